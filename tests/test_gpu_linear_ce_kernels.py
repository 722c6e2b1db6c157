"""Each kernel of the gradients of the loss over a vocabulary against 64 bits on the GPU: the logits, d_h and d_w in tiles of 256, 192 and 128 (one and two workgroups on a compute unit), whole and in
slices of the contraction; at sizes whose tiles, slabs and pieces end anywhere, with tokens that have no target.

Bounds element by element, as for small sizes (test_gpu_linear_ce.py): dz off by its rounding to bf16 and its exponential's error, a gradient by these times the other operand, by its fp32 sum
(n / 4 + 16 roundings of the sum of magnitudes) and its own rounding.  A logit's sum of dim products is off by (dim / 4 + 16) 2^-24 of its magnitude as there, or, where that is less, by 2 sqrt(dim) + 16: eight
roundings of each of dim / 32 matrix instructions, independent ones, add as roots of squares, 1.4 sqrt(dim)."""
import pytest

import test_gpu_linear_ce as many

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ah = many.ah

U32, BF16 = 2.0 ** -24, 2.0 ** -8

# tokens, dim, vocabulary; of the logits, d_h and d_w: the tile (128 alone: negative) and whether some tiles are cut into slices
SIZES = [
    (1301, 3001, 101, (-128, 0), (128, 0), (-128, 0)), (1299, 5999, 103, (-128, 0), (192, 0), (-128, 0)), (301, 6001, 8003, (-128, 0), (192, 1), (256, 0)),
    (2501, 3499, 101, (-128, 0), (256, 0), (-128, 1)), (1301, 3503, 8005, (256, 0), (256, 1), (256, 0)), (9, 6001, 701, (-128, 0), (-128, 0), (128, 0)), (9, 1501, 6003, (-128, 0), (-128, 1), (192, 0)),
    (8003, 6001, 303, (-128, 0), (256, 0), (192, 1)), (8003, 501, 10003, (256, 0), (-128, 0), (256, 1)), (1301, 9, 3003, (128, 0), (-128, 1), (-128, 0)), (1301, 9, 6003, (192, 0), (-128, 1), (-128, 0)),
    (3601, 9, 2503, (256, 0), (-128, 1), (-128, 1)), (4096, 4096, 4096, (256, 0), (256, 0), (256, 0)), (2050, 4099, 4101, (192, 0), (192, 0), (192, 0)),
    (17635, 3, 27407, (256, 0), (128, 1), (-128, 0)), (4037, 5, 71731, (256, 0), (-128, 1), (128, 1)),
    (8, 1030, 70, (-128, 0), (-128, 0), (0, 0)),
]


def check_plan(ah, T, D, V, wanted):
    got = [ah.adahop_debug_linear_ce_plan(T, V, D, i) for i in range(3)]
    assert [(-t if alone else t, int(slices > 1)) for t, alone, slices in got] == list(wanted), f"other kernels than this test is of: {got}"


def within(got, want, bound, what):
    over = ((got.double() - want).abs() / bound).max().item()
    assert over <= 1.0, f"{what}: {over:.2f} times what is allowed"


def compare(ah, gen, h, w, y, scale=0.7, z_loss=1e-3):
    """Loss and gradients of these tokens, d_w in either type with something added, outputs among other memory."""
    (T, D), V = h.shape, w.shape[0]
    g, add = torch.randn(T, generator=gen, device="cuda"), torch.randn(V, D, generator=gen, device="cuda")
    h64, w64 = h.double(), w.double()
    turned = w64.t().contiguous()
    z = (h64 @ turned).mul_(scale)
    l64 = torch.logsumexp(z, 1)
    lse = l64.float()
    ez = (h64.abs() @ turned.abs()).mul_((min(D / 4, 2 * D ** 0.5) + 16) * U32 * scale)
    f = ah.adahop_linear_ce(h, w, y, logit_scale=scale, z_loss=z_loss)
    e_lse = ez.amax(1) + (160 + V / 2048) * U32 + 2 * U32 * l64.abs()
    within(f["lse"], l64, e_lse, "lse")
    there = y >= 0
    at = z.gather(1, y.clamp(min=0)[:, None])[:, 0]
    loss = torch.where(there, l64 - at + z_loss * l64 * l64, torch.zeros_like(l64))
    within(f["loss"], loss, e_lse + ez.amax(1) + 2 * z_loss * l64.abs() * e_lse + 4 * U32 * (loss.abs() + l64.abs() + z_loss * l64 * l64), "loss")
    l64 = lse.double()[:, None]
    z.sub_(l64)
    e = ez.add_(z.abs().mul_(2 * U32)).add_(16 * U32)       # of exp(z - lse), relative, and of its factor
    p = z.exp_().mul_(1 + 2 * z_loss * l64)
    e.mul_(p.abs())
    p[there.nonzero()[:, 0], y[there]] -= 1.0
    gain = torch.where(there, g.double() * scale, torch.zeros_like(g, dtype=torch.float64))[:, None]
    dz, size = p.mul_(gain), e.mul_(gain.abs() * (1 + BF16))
    e_dz = size.add_(dz.abs() * BF16)
    how = dict(logit_scale=scale, z_loss=z_loss)
    for target, got_bf16 in (("d_h", True), ("d_w", True), ("d_w", False)):
        n = V if target == "d_h" else T
        a, ea, other = (dz, e_dz, w64) if target == "d_h" else (dz.t().contiguous(), e_dz.t().contiguous(), h64)
        want = a @ other
        bound = ea @ other.abs() + (a.abs() @ other.abs()) * ((n / 4 + 16) * U32)
        if target == "d_w":
            more = add.to(torch.bfloat16) if got_bf16 else add
            want += more.double()
            bound += 2 * U32 * more.double().abs()
            room = torch.full((V + 1, D + 3), 7.0, dtype=torch.bfloat16 if got_bf16 else torch.float32, device="cuda")
            out = ah.adahop_linear_ce_backward(h, w, y, lse, g, add=more, d_w=room[:V, :D], want_h=False, **how)["d_w"]
        else:
            room = torch.full((T + 1, D + 3), 7.0, dtype=torch.bfloat16, device="cuda")
            out = ah.adahop_linear_ce_backward(h, w, y, lse, g, d_h=room[:T, :D], want_w=False, **how)["d_h"]
        bound += 2 * U32 * want.abs()
        if got_bf16:
            bound = bound + BF16 * (want.abs() + bound)
        within(out, want, bound + 1e-37, target)
        assert bool((room[-1] == 7).all()) and bool((room[:, D:] == 7).all())
        if target == "d_h":
            assert not out[y < 0].any()
    both = ah.adahop_linear_ce_backward(h, w, y, lse, g, **how)
    assert torch.equal(both["d_h"], ah.adahop_linear_ce_backward(h, w, y, lse, g, want_w=False, **how)["d_h"])
    assert torch.equal(both["d_w"], ah.adahop_linear_ce_backward(h, w, y, lse, g, want_h=False, **how)["d_w"])


def targets(gen, T, V):
    y = torch.randint(0, V, (T,), generator=gen, device="cuda")
    y[torch.rand(T, generator=gen, device="cuda") < 0.2] = -100
    y[0], y[T - 1] = V - 1, 0
    return y


@pytest.mark.parametrize("T,D,V,logits,d_h,d_w", SIZES)
def test_against_64_bits(ah, T, D, V, logits, d_h, d_w):
    check_plan(ah, T, D, V, (logits, d_h, d_w))
    gen = torch.Generator(device="cuda").manual_seed(T * 5 + D + V)
    many.say("gradient kernels", T, D, V)
    h, w = torch.randn(T, D, generator=gen, device="cuda").to(torch.bfloat16), torch.randn(V, D, generator=gen, device="cuda").mul_(D ** -0.5).to(torch.bfloat16)
    compare(ah, gen, h, w, targets(gen, T, V))
