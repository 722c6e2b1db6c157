"""The training operators on a stream that the call names: where the memory comes from, who gets it next, and what is refused."""
import pytest

import test_gpu_training_ops as small

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ah = small.ah

ROWS, COLS = 1024, 2048


def tensors(out):
    for v in out.values() if isinstance(out, dict) else (out,):
        yield from (t for t in (v if isinstance(v, tuple) else (v,)) if t is not None)


def same(a, b):
    a, b = list(tensors(a)), list(tensors(b))
    return len(a) == len(b) and all(torch.equal(p, q) for p, q in zip(a, b))


def the_calls(ah):
    """Name -> call(stream), the inputs ready."""
    x, y, d, w, _ = small.operands(ROWS, COLS)
    G = d[:, :136].contiguous()
    f = ah.adahop_block_norm(x, y, w_post=w, w_pre=w, gate=w, keep="ckpt8")
    back = (d, y, f["ckpt_s"], f["ckpt_y"], f["rstd_pre"], f["rstd_post"])
    calls = {
        "pack": lambda s: ah.adahop_ckpt8_pack(x, stream=s),
        "unpack": lambda s: ah.adahop_ckpt8_unpack(f["ckpt_s"], stream=s),
        "swiglu": lambda s: ah.adahop_swiglu(x, y, keep8=True, stream=s),
        "swiglu backward": lambda s: ah.adahop_swiglu_backward(x, y, d, stream=s),
        "norm": lambda s: ah.adahop_block_norm(x, y, w_post=w, w_pre=w, gate=w, keep="ckpt8", stream=s),
        "norm backward": lambda s: ah.adahop_block_norm_backward(*back, w_post=w, w_pre=w, gate=w, stream=s),
        "wgrad": lambda s: ah.adahop_ckpt8_wgrad(G, f["ckpt_s"], stream=s),
    }
    torch.cuda.synchronize()
    return calls


def spans(ts):
    return [(t.data_ptr(), t.data_ptr() + max(t.untyped_storage().nbytes() - t.storage_offset() * t.element_size(), 1)) for t in ts]


def overlap(a, b):
    return any(p < s and r < q for p, q in a for r, s in b)


NAMES = ["pack", "unpack", "swiglu", "swiglu backward", "norm", "norm backward", "wgrad"]


@pytest.mark.parametrize("name", NAMES)
def test_memory_of_a_named_stream(ah, name):
    """Outputs lie in memory that no queued work of the current stream can still use, and that the current stream does not get while the call's stream is not done."""
    call = the_calls(ah)[name]
    want = call(None)
    other = torch.cuda.Stream()
    small.say("memory of a named stream:", name)
    freed = [torch.empty_like(t) for t in tensors(want)]
    were = spans(freed)
    del freed                                       # the current stream's earlier work may still read or write these
    torch.cuda._sleep(20_000_000)
    got = call(other)
    assert not overlap(spans(tensors(got)), were)
    lost = spans(tensors(got))
    other.synchronize()
    torch.cuda.synchronize()
    assert same(got, want)
    del got                                         # dropped while its stream is busy:
    with torch.cuda.stream(other):
        torch.cuda._sleep(20_000_000)
    dropped = spans(tensors(call(other)))
    mine = [torch.empty_like(t) for _ in range(4) for t in tensors(want)]
    assert not overlap(spans(mine), dropped + lost)
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", NAMES)
def test_outputs_read_on_the_current_stream(ah, name):
    """Dropped while the current stream still reads them, they are not handed to the next call on their own stream."""
    call = the_calls(ah)[name]
    want = call(None)
    other = torch.cuda.Stream()
    small.say("outputs read on the current stream:", name)
    got = call(other)
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda._sleep(50_000_000)
    copies = [t.clone() for t in tensors(got)]      # queued behind the sleep
    were = spans(tensors(got))
    del got
    more = call(other)
    assert not overlap(spans(tensors(more)), were)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(copies, tensors(want))) and same(more, want)


@pytest.mark.parametrize("name", NAMES)
def test_bare_handles(ah, name):
    """The current stream's is as good as none; another stream's needs all memory given."""
    call = the_calls(ah)[name]
    want = call(None)
    other = torch.cuda.Stream()
    small.say("bare handles:", name)
    assert same(call(torch.cuda.current_stream().cuda_stream), want)
    with pytest.raises(ValueError, match="bare handle"):
        call(other.cuda_stream)
    with torch.cuda.stream(other):
        assert same(call(other.cuda_stream), want)
        with pytest.raises(ValueError, match="bare handle"):
            call(torch.cuda.default_stream().cuda_stream)
    for stream in ("0", 1.5, object()):
        with pytest.raises(TypeError, match="stream"):
            call(stream)
    torch.cuda.synchronize()


def test_bare_handles_with_all_memory_given(ah):
    x, y, d, w, G = small.operands(ROWS, COLS)
    like = lambda o: {k: tuple(torch.empty_like(t) for t in v) if isinstance(v, tuple) else torch.empty_like(v) for k, v in o.items() if v is not None}  # noqa: E731
    want = ah.adahop_block_norm(x, y, w_post=w, w_pre=w, keep="ckpt8")
    back = (d, y, want["ckpt_s"], want["ckpt_y"], want["rstd_pre"], want["rstd_post"])
    want_b = ah.adahop_block_norm_backward(*back, w_post=w, w_pre=w)
    want_c = ah.adahop_ckpt8_wgrad(G, want["ckpt_s"])
    out, out_b, out_c = like(want), like(want_b), torch.empty_like(want_c)
    scratch = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    h = other.cuda_stream
    small.say("bare handles, memory given")
    got = ah.adahop_block_norm(x, y, w_post=w, w_pre=w, **out, stream=h)
    got_b = ah.adahop_block_norm_backward(*back, w_post=w, w_pre=w, **out_b, workspace=scratch, stream=h)
    with pytest.raises(ValueError, match="bare handle"):
        ah.adahop_ckpt8_wgrad(G, want["ckpt_s"], Cout=out_c, stream=h)
    got_c = ah.adahop_ckpt8_wgrad(G, want["ckpt_s"], Cout=out_c, workspace=scratch, stream=h)
    other.synchronize()
    assert same(got, want) and same(got_b, want_b) and torch.equal(got_c, want_c)


def test_the_stream_is_taken(ah):
    """A call waits for what is queued on its stream, and the current stream is what it was."""
    x, y, d, w, _ = small.operands(ROWS, COLS)
    want = ah.adahop_ckpt8_pack(x * 2)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    now = torch.cuda.current_stream()
    small.say("the stream is taken")
    with torch.cuda.stream(other):
        torch.cuda._sleep(20_000_000)
        x.mul_(2)
    got = ah.adahop_ckpt8_pack(x, stream=other)
    assert torch.cuda.current_stream() == now
    other.synchronize()
    assert same({"k": got}, {"k": want})
