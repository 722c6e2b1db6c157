"""Gradients of the loss over a vocabulary for few tokens, where d_w has a kernel of its own (up to eight of them), at both sides of that and at odd sizes, against 64 bits: bounds as for
any number of tokens."""
import numpy as np
import pytest

import test_gpu_linear_ce as many

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ah = many.ah


@pytest.mark.parametrize("T", [1, 2, 5, 8, 9])
@pytest.mark.parametrize("D,V", [(1, 1), (5, 33), (64, 8), (1030, 70), (2056, 321)])
def test_gradients_of_few_tokens(ah, T, D, V):
    many.say("few tokens", T, D, V)
    c = many.Case(T, D, V, z_loss=1e-3, logit_scale=0.7, ignored=0.3 if T > 2 else 0.0)
    h, w, t = many.up(c.h, pad=3), many.up(c.w), torch.from_numpy(c.targets).cuda()
    lse, g = torch.from_numpy(c.lse32).float().cuda(), torch.from_numpy(c.d_loss).float().cuda()
    before = many.bf16(np.random.default_rng(3).normal(size=(V, D)))
    for dtype in (torch.float32, torch.bfloat16):
        room = torch.full((V + 1, D + 3), 7, dtype=dtype, device="cuda")
        out = ah.adahop_linear_ce_backward(h, w, t, lse, g, d_w=room[:V, :D], **c.options)
        torch.cuda.synchronize()
        c.gradients((out["d_h"], False), (out["d_w"], dtype == torch.float32))
        assert bool((room[V:] == 7).all()) and bool((room[:, D:] == 7).all())
    for dtype in (torch.float32, torch.bfloat16):  # what is added: of either type, and the result itself
        add = torch.from_numpy(before).to(dtype).cuda()
        out = ah.adahop_linear_ce_backward(h, w, t, lse, g, add=add, want_h=False, **c.options)
        c.gradients(None, (out["d_w"], True), add=before)
    d_w = torch.from_numpy(before).float().cuda()
    ah.adahop_linear_ce_backward(h, w, t, lse, g, d_w=d_w, add=d_w, want_h=False, **c.options)
    c.gradients(None, (d_w, True), add=before)


@pytest.mark.parametrize("T", [1, 8])
def test_no_target_among_few_tokens(ah, T):
    """Nothing but what is added, whatever the tokens hold."""
    many.say("no target", T)
    h = torch.full((T, 40), float("nan"), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(50, 40, dtype=torch.bfloat16, device="cuda")
    add = torch.randn(50, 40, device="cuda")
    out = ah.adahop_linear_ce_backward(h, w, torch.full((T,), -1, device="cuda"), torch.zeros(T, device="cuda"), add=add)
    assert torch.equal(out["d_w"], add) and not out["d_h"].any()


def test_few_tokens_from_a_graph(ah):
    """Replayed with other targets among other work, every time the eager result."""
    many.say("graph")
    draw = torch.Generator(device="cuda").manual_seed(2)
    h, w = (torch.randn(n, 96, generator=draw, device="cuda").to(torch.bfloat16) for n in (6, 500))
    targets = torch.zeros(6, dtype=torch.int64, device="cuda")
    ah.adahop_prepare_device()

    def step():
        f = ah.adahop_linear_ce(h, w, targets)
        return ah.adahop_linear_ce_backward(h, w, targets, f["lse"])
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        targets.copy_(torch.randint(-2, 500, (6,), generator=draw, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        for k in want:
            assert torch.equal(out[k], want[k]), (i, k)
