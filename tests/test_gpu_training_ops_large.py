"""The training operators where runs of rows have several rows, rows are wider than a workgroup, and offsets pass 32 bits."""
import pytest

import test_gpu_training_ops as small

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ah = small.ah


@pytest.mark.parametrize("rows,cols", [(2100, 1032), (1300, 8264), (4200, 300)])
@pytest.mark.parametrize("gate", [None, "vector", 3, 7, 1, 700])
@pytest.mark.parametrize("kept", [True, False])
def test_block_norm_backward_of_many_rows(ah, rows, cols, gate, kept):
    """Runs of several rows, beside each other in a workgroup or in strips, and groups of rows that end within them."""
    small.test_block_norm_backward(ah, rows, cols, gate, kept, False, False, 0)


class Far:
    """Tensors whose rows lie more than 2^31 elements apart, in one allocation."""

    def __init__(self):
        self.room = torch.empty(2 ** 33 + 2 ** 20, dtype=torch.int16, device="cuda")
        self.used = 0

    def like(self, t, apart):
        view = self.room.view(t.dtype) if t.element_size() != 1 else self.room.view(torch.uint8)
        at = self.used // t.element_size()
        self.used += (t.shape[1] * t.element_size() + 255) // 256 * 256
        return view[at:].as_strided(t.shape, (apart, 1))

    def of(self, t, apart):
        return self.like(t, apart).copy_(t)


def test_offsets_beyond_32_bits(ah):
    """Three rows, the last beginning more than 2^32 elements after the first: the same bits as from rows beside each other."""
    rows, cols = 3, 1000
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, y, d_s, d_h = (torch.randn(rows, cols, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(4))
    w = torch.randn(cols, generator=gen, device="cuda").to(torch.bfloat16)
    far, apart = Far(), 2 ** 31 + 2 ** 20
    wide8 = lambda k: (far.like(k[0], 2 ** 32 + 2 ** 20), far.like(k[1], 2 ** 32 + 2 ** 20))  # noqa: E731
    same = lambda a, b: all(torch.equal(p, q) for p, q in zip(a, b))  # noqa: E731
    small.say("far rows")
    near = ah.adahop_block_norm(x, y, w_post=w, w_pre=w, gate=w, keep="ckpt8")
    fx, fy = far.of(x, apart), far.of(y, apart)
    got = ah.adahop_block_norm(fx, fy, w_post=w, w_pre=w, gate=w, keep="ckpt8", s=far.like(x, apart), h=far.like(x, apart),
                               ckpt_y=wide8(near["ckpt_y"]), ckpt_s=wide8(near["ckpt_s"]))
    assert torch.equal(got["s"], near["s"]) and torch.equal(got["h"], near["h"])
    assert same(got["ckpt_y"], near["ckpt_y"]) and same(got["ckpt_s"], near["ckpt_s"])
    more = dict(w_post=w, w_pre=w, gate=w)
    near_b = ah.adahop_block_norm_backward(d_s, d_h, near["ckpt_s"], near["ckpt_y"], near["rstd_pre"], near["rstd_post"], **more)
    got_b = ah.adahop_block_norm_backward(far.of(d_s, apart), far.of(d_h, apart), got["ckpt_s"], got["ckpt_y"], near["rstd_pre"], near["rstd_post"],
                                          d_x=far.like(x, apart), d_y=far.like(x, apart), **more)
    assert all(torch.equal(got_b[n], near_b[n]) for n in near_b)
    near_a = ah.adahop_swiglu(x, y, keep8=True)
    got_a = ah.adahop_swiglu(fx, fy, a=far.like(x, apart), ckpt_g=wide8(near_a["ckpt_g"]), ckpt_u=wide8(near_a["ckpt_u"]))
    assert torch.equal(got_a["a"], near_a["a"]) and same(got_a["ckpt_g"], near_a["ckpt_g"]) and same(got_a["ckpt_u"], near_a["ckpt_u"])
    near_d = ah.adahop_swiglu_backward(near_a["ckpt_g"], near_a["ckpt_u"], d_s, a=ah.adahop_ckpt8_empty(rows, cols))
    got_d = ah.adahop_swiglu_backward(got_a["ckpt_g"], got_a["ckpt_u"], far.of(d_s, apart), d_g=far.like(x, apart), d_u=far.like(x, apart),
                                      a=wide8(near_d["a"]))
    assert torch.equal(got_d["d_g"], near_d["d_g"]) and torch.equal(got_d["d_u"], near_d["d_u"]) and same(got_d["a"], near_d["a"])
    near_k = ah.adahop_ckpt8_pack(x)
    got_k = ah.adahop_ckpt8_pack(fx, out=wide8(near_k))
    assert same(got_k, near_k)
    assert torch.equal(ah.adahop_ckpt8_unpack(got_k, out=far.like(x, apart)), ah.adahop_ckpt8_unpack(near_k))


def test_weight_gradient_of_far_rows(ah):
    """Output gradient, checkpoint, result and what is added with rows 2^24 elements apart: the last token's begins beyond 2^32 bytes."""
    tokens, d_out, d_in, apart = 300, 264, 520, 2 ** 24
    gen = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    G, x8, add = r(tokens, d_out).to(torch.bfloat16), ah.adahop_ckpt8_pack(r(tokens, d_in).to(torch.bfloat16)), r(d_out, d_in).to(torch.bfloat16)
    far = Far()
    small.say("far rows of a weight gradient")
    want = ah.adahop_ckpt8_wgrad(G, x8, add=add, c_bf16=True)
    got = ah.adahop_ckpt8_wgrad(far.of(G, apart), (far.of(x8[0], apart), far.of(x8[1], apart)), add=far.of(add, apart), Cout=far.like(add, apart))
    assert torch.equal(got, want)


@pytest.mark.parametrize("rows,cols", [(600, 1032), (600, 8264), (600, 4096)])
def test_workspaces_of_a_stream_of_its_own(ah, rows, cols):
    """Calls that name a stream bring their scratch along; the bits are those of the current stream's calls."""
    x, y, d, w, G = small.operands(rows, cols)
    f = ah.adahop_block_norm(x, y, w_post=w, w_pre=w, gate=w, keep="ckpt8")
    args = (d, d, f["ckpt_s"], f["ckpt_y"], f["rstd_pre"], f["rstd_post"])
    want = ah.adahop_block_norm_backward(*args, w_post=w, w_pre=w, gate=w)
    grad = ah.adahop_ckpt8_wgrad(G, f["ckpt_s"])
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    small.say("a stream of its own", rows, cols)
    got = ah.adahop_block_norm_backward(*args, w_post=w, w_pre=w, gate=w, stream=other)
    again = ah.adahop_ckpt8_wgrad(G, f["ckpt_s"], stream=other)
    other.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in want) and torch.equal(again, grad)
