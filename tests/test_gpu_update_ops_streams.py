"""The loss over a vocabulary and the updates of weights on streams, in graphs, beside each other, and in workspaces that hold anything."""
import pytest

import test_gpu_training_ops_streams as streams

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ah = streams.ah
tensors, same, spans, overlap = streams.tensors, streams.same, streams.spans, streams.overlap


def say(*a):
    print("[case]", *a, flush=True)


def inputs(T=300, D=128, V=1000, m=200, n=330, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    return {"h": randn(T, D).to(torch.bfloat16), "w": (randn(V, D) * D ** -0.5).to(torch.bfloat16), "y": torch.where(randn(T) > 1.0, -100, y), "d": randn(T),
            "g": randn(m, n), "weight": randn(m, n) * 0.02, "momentum": randn(m, n)}


def the_calls(ah, x):
    lse = ah.adahop_linear_ce(x["h"], x["w"], x["y"])["lse"]
    calls = {
        "loss": lambda **k: ah.adahop_linear_ce(x["h"], x["w"], x["y"], z_loss=1e-3, **k),
        "loss backward": lambda **k: ah.adahop_linear_ce_backward(x["h"], x["w"], x["y"], lse, x["d"], **k),
        "orthogonalize": lambda **k: ah.adahop_orthogonalize(x["g"], **k),
        "update": lambda **k: ah.adahop_muon_update(x["weight"], x["g"], x["momentum"], 0.02, w_out=torch.empty_like(x["weight"]), momentum_out=torch.empty_like(x["momentum"]), **k),
    }
    torch.cuda.synchronize()
    return calls


NAMES = ["loss", "loss backward", "orthogonalize", "update"]


@pytest.mark.parametrize("name", NAMES)
def test_memory_of_a_named_stream(ah, name):
    """Outputs and workspaces lie in memory that no queued work of the current stream can still use, and that the current stream does not get while the call's stream is not done."""
    call = the_calls(ah, inputs())[name]
    want = call()
    other = torch.cuda.Stream()
    say("memory of a named stream:", name)
    torch.cuda._sleep(20_000_000)
    got = call(stream=other)
    if name != "update":                            # whose outputs are the caller's
        freed = spans(tensors(want))
        assert not overlap(spans(tensors(got)), freed)
    other.synchronize()
    torch.cuda.synchronize()
    assert same(got, want)
    with torch.cuda.stream(other):
        torch.cuda._sleep(20_000_000)
    got = call(stream=other)
    junk = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(8)]      # the current stream's, while the other is not done
    torch.cuda.synchronize()
    assert same(got, want) and len(junk) == 8


@pytest.mark.parametrize("name", NAMES)
def test_bare_handles(ah, name):
    call = the_calls(ah, inputs())[name]
    want = call()
    other = torch.cuda.Stream()
    say("bare handles:", name)
    assert same(call(stream=torch.cuda.current_stream().cuda_stream), want)
    with pytest.raises(ValueError, match="bare handle"):
        call(stream=other.cuda_stream)
    for stream in ("0", 1.5, object()):
        with pytest.raises(TypeError, match="stream"):
            call(stream=stream)
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", NAMES)
def test_workspaces_of_any_content(ah, name):
    """What lies in the workspace before, NaN everywhere here, is not seen in the result."""
    say("workspace:", name)
    for x in (inputs(), inputs(T=5, D=72, V=131, m=70, n=1500), inputs(T=777, D=40, V=2050, m=1500, n=64)):
        call = the_calls(ah, x)[name]
        want = call()
        for byte in (0xFF, 0x7F):
            got = call(workspace=torch.full((1 << 27,), byte, dtype=torch.uint8, device="cuda"))
            torch.cuda.synchronize()
            assert same(got, want)
        with pytest.raises(ah.AdahopError):
            call(workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
        with pytest.raises(ValueError):
            call(workspace=torch.empty(1 << 20, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("m,n", [(200, 330), (1500, 600)])
def test_a_step_replays_from_a_graph(ah, m, n):
    """Loss, gradients and updates of both weights, captured once and replayed on other inputs, with eager work between the replays.  One workspace serves all calls."""
    ah.adahop_prepare_device()
    x = inputs(m=m, n=n)
    V, D = x["w"].shape
    need = 1 << 28
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    T = x["h"].shape[0]
    out = {k: torch.empty(T, device="cuda") for k in ("loss", "lse")}
    d_h, d_w = torch.empty_like(x["h"]), torch.empty(V, D, device="cuda")
    head, mom_head, copy = x["w"].float(), torch.zeros(V, D, device="cuda"), torch.empty_like(x["w"])

    def step():
        ah.adahop_linear_ce(x["h"], x["w"], x["y"], workspace=ws, **out)
        ah.adahop_linear_ce_backward(x["h"], x["w"], x["y"], out["lse"], x["d"], d_h=d_h, d_w=d_w, workspace=ws)
        ah.adahop_muon_update(head, d_w, mom_head, 0.02, w_bf16=copy, workspace=ws)
        ah.adahop_muon_update(x["weight"], x["g"], x["momentum"], 0.02, weight_decay=0.1, workspace=ws)
        return [t.clone() for t in (out["loss"], d_h, d_w, head, mom_head, copy, x["weight"], x["momentum"])]

    def start(seed):
        new = inputs(m=m, n=n, seed=seed)
        for k in x:
            x[k].copy_(new[k])
        head.copy_(x["w"].float())
        mom_head.zero_()
        torch.cuda.synchronize()
    step()
    start(1)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            captured = step()
    torch.cuda.synchronize()
    for seed in (2, 3, 4):
        say("graph replay", m, n, seed)
        start(seed)
        want = step()
        torch.cuda.synchronize()
        start(seed)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want))


def test_two_calls_at_once(ah):
    """On two streams, each with a workspace of its own."""
    say("two at once")
    xs = [inputs(T=900, D=256, V=5000, m=700, n=900, seed=s) for s in (5, 6)]
    calls = [the_calls(ah, x) for x in xs]
    want = [{k: c[k]() for k in NAMES} for c in calls]
    torch.cuda.synchronize()
    both = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = [{k: c[k](stream=s) for k in NAMES} for c, s in zip(calls, both)]
        torch.cuda.synchronize()
        assert all(same(g[k], w[k]) for g, w in zip(got, want) for k in NAMES)
