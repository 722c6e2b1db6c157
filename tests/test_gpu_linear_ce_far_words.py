"""The loss over a vocabulary and its gradients where a token's probability lies on four words at known places: the first, the last, two of the last hundredth, whose rows lie past 2^31
elements where the vocabulary is large.  A word that is left out, or another's in its place, moves lse by some 0.2 and d_h by a fifth of itself.

Bounds: a logit is a sum of dim products, off by (dim / 4 + 16) 2^-24 of the sum m of their magnitudes; lse by the largest such error, its sums' 160 * 2^-24 + 2 * 2^-24 |lse| as for
small sizes (test_gpu_linear_ce.py) and, where up to eight tokens' words go by 2048 waves, the V / 2048 additions of a wave.  d_h and d_w as there; d_h's sum over the vocabulary is of V / 32 additions in a row at
most, whose roundings, independent ones of 2^-24 of the sum, add as roots of squares: three times sqrt(2^20 / 32) = 181 and 32 within an addition."""
import pytest

import test_gpu_linear_ce as many

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ah = many.ah

U32, BF16 = 2.0 ** -24, 2.0 ** -8


@pytest.mark.parametrize("T,D,V", [(3, 2056, 1050001), (8, 2048, 1050007), (8, 8200, 3000), (4, 8200, 3001), (1, 512, 70000), (600, 1024, 30000), (1700, 256, 9000), (30, 2056, 1050001)])
def test_words_that_count(ah, T, D, V):
    many.say("far words", T, D, V)
    gen = torch.Generator(device="cuda").manual_seed(T + D + V)
    h = torch.randn(T, D, generator=gen, device="cuda").to(torch.bfloat16)
    w = torch.empty(V, D, dtype=torch.bfloat16, device="cuda")
    for i in range(0, V, 1 << 16):
        w[i:i + (1 << 16)] = torch.randn(min(1 << 16, V - i), D, generator=gen, device="cuda") * 1e-3
    # token t's words: from either end on, and two of the last hundredth (or thereabouts, where tokens are many)
    t = torch.arange(T, device="cuda")
    last = max(V // 100, 3 * T)
    words = torch.stack((t, V - 1 - t, V - T - 1 - t * ((last - T) // 2 // T), V - last - 1 - t), 1)
    assert len(words.unique()) == 4 * T
    for k in range(4):
        w[words[:, k]] = (h.double() * (16.0 / h.double().square().sum(1, keepdim=True))).to(torch.bfloat16)
    y = words[t, t % 4].clone()
    y[T // 2] = V // 3                                   # one whose target is none of them
    z_loss, g = 1e-4, torch.rand(T, generator=gen, device="cuda") + 0.5

    parts, mag = [], torch.zeros(T, dtype=torch.float64, device="cuda")
    h64 = h.double()
    for i in range(0, V, 1 << 15):
        turned = w[i:i + (1 << 15)].double().t().contiguous()
        parts.append(torch.logsumexp(h64 @ turned, 1))
        mag = torch.maximum(mag, (h64.abs() @ turned.abs()).amax(1))
    lse = torch.logsumexp(torch.stack(parts), 0)
    ez = (D / 4 + 16) * U32 * mag
    e_lse = ez + (160 + V / 2048) * U32 + 2 * U32 * lse.abs()
    out = ah.adahop_linear_ce(h, w, y, z_loss=z_loss)
    assert ((out["lse"].double() - lse).abs() <= e_lse).all(), ((out["lse"].double() - lse).abs() / e_lse).max()
    at = (h64 * w[y].double()).sum(1)
    loss = lse - at + z_loss * lse * lse
    e_loss = e_lse + ez + 2 * z_loss * lse.abs() * e_lse + 4 * U32 * (loss.abs() + lse.abs() + z_loss * lse * lse)
    assert ((out["loss"].double() - loss).abs() <= e_loss).all()

    given = lse.float()
    factor = (1 + 2 * z_loss * given.double())[:, None]
    back = ah.adahop_linear_ce_backward(h, w, y, given, g, z_loss=z_loss, d_w_bf16=True)
    want, size = (torch.zeros(T, D, dtype=torch.float64, device="cuda") for _ in range(2))
    for i in range(0, V, 1 << 15):
        part = w[i:i + (1 << 15)].double()
        z = h64 @ part.t().contiguous()
        p = torch.exp(z - given.double()[:, None]) * factor
        e = p * (ez[:, None] + 2 * U32 * (z - given.double()[:, None]).abs() + 16 * U32)
        here = ((y >= i) & (y < i + len(part))).nonzero()[:, 0]
        p[here, y[here] - i] -= 1.0
        dz, e = p * g.double()[:, None], e * g.double()[:, None]
        e = e * (1 + BF16) + BF16 * dz.abs()
        want += dz @ part
        size += (e + 576 * U32 * dz.abs()) @ part.abs()
        if i == 0 or i + (2 << 15) >= V or ((words >= i) & (words < i + len(part))).any():
            exact = dz.t().contiguous() @ h64
            bound = e.t().contiguous() @ h64.abs() + (T / 4 + 16) * U32 * (dz.abs().t().contiguous() @ h64.abs())
            bound = bound + BF16 * (exact.abs() + bound) + 2 * U32 * exact.abs() + 1e-37
            over = ((back["d_w"][i:i + len(part)].double() - exact).abs() / bound).max().item()
            assert over <= 1.0, (i, over)
    bound = size + BF16 * (want.abs() + size) + 2 * U32 * want.abs() + 1e-37
    over = ((back["d_h"].double() - want).abs() / bound).max().item()
    assert over <= 1.0, over
