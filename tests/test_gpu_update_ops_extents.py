"""The loss over a vocabulary and the updates at the limits of what they accept: 2^21 tokens, words or features, rows of h and w 2^22 elements apart, rows of a matrix 2^26 apart."""
import pytest

import test_gpu_linear_ce_kernels as loss
import test_gpu_newton_schulz_kernels as updates

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ah = loss.ah

MOST = 1 << 21


@pytest.mark.parametrize("T,D,V", [(MOST, 8, 300), (MOST, 3, 7), (300, 16, MOST), (5, 24, MOST), (20, MOST, 40), (3, MOST, 9), (300, MOST - 8, 5)])
def test_loss_of_the_largest_extents(ah, T, D, V):
    gen = torch.Generator(device="cuda").manual_seed(T + D + V)
    loss.many.say("largest extents", T, D, V)
    h, w = torch.randn(T, D, generator=gen, device="cuda").to(torch.bfloat16), torch.randn(V, D, generator=gen, device="cuda").mul_(D ** -0.5).to(torch.bfloat16)
    loss.compare(ah, gen, h, w, loss.targets(gen, T, V))


def far_apart(x, ld, dtype):
    """x in rows `ld` elements apart, what lies between them never written"""
    v = torch.empty(x.shape[0] * ld, dtype=dtype, device="cuda").view(x.shape[0], ld)[:, :x.shape[1]]
    v.copy_(x)
    return v


@pytest.mark.parametrize("T,D,V", [(300, 64, 520), (520, 72, 300), (6, 64, 300)])
def test_loss_of_rows_far_apart(ah, T, D, V):
    gen = torch.Generator(device="cuda").manual_seed(T + D + V)
    loss.many.say("rows far apart", T, D, V)
    ld = (1 << 22) - 8
    h, w = far_apart(torch.randn(T, D, generator=gen, device="cuda"), ld, torch.bfloat16), far_apart(torch.randn(V, D, generator=gen, device="cuda").mul_(D ** -0.5), ld, torch.bfloat16)
    y = loss.targets(gen, T, V)
    loss.compare(ah, gen, h, w, y)
    torch.cuda.empty_cache()
    f = ah.adahop_linear_ce(h.contiguous(), w.contiguous(), y)
    back = ah.adahop_linear_ce_backward(h.contiguous(), w.contiguous(), y, f["lse"])
    far = ah.adahop_linear_ce_backward(h, w, y, f["lse"], d_h=far_apart(h, ld, torch.bfloat16), d_w=far_apart(w, ld, torch.bfloat16))
    assert torch.equal(far["d_h"], back["d_h"]) and torch.equal(far["d_w"], back["d_w"].to(torch.bfloat16))


@pytest.mark.parametrize("m,n", [(140, 150), (140, 6000), (200, 100), (140, 40)])
def test_matrices_of_rows_far_apart(ah, m, n):
    """Tiles of 64, of 128, the iterate as two numbers, and slices that another kernel joins: the same bits as close together."""
    loss.many.say("matrices of rows far apart", m, n)
    g = updates.matrix(m, n)
    want = ah.adahop_orthogonalize(g, dtype=torch.float32)
    updates.check(want, updates.exact(g.double(), 5))
    ld = (1 << 26) - 1
    far = far_apart(g, ld, torch.float32)
    out = far_apart(torch.zeros_like(g), ld, torch.float32)
    ah.adahop_orthogonalize(far, out=out)
    assert torch.equal(out, want)
    del out
    mom, w = torch.ones(m, n, device="cuda"), torch.randn(m, n, device="cuda")
    far_w = far_apart(w, ld, torch.float32)
    copy = far_apart(torch.zeros_like(w), ld, torch.bfloat16)
    ah.adahop_muon_update(far_w, far, mom.clone(), 0.1, w_bf16=copy)
    ah.adahop_muon_update(w, g, mom, 0.1)
    assert torch.equal(far_w, w) and torch.equal(copy, w.to(torch.bfloat16))
    del far, far_w, copy
    torch.cuda.empty_cache()
