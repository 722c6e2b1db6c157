"""Each kernel of the weight gradient from an 8-bit checkpoint against a product in 64 bits: tiles of 256 and of 128 columns, the latter with one workgroup's tokens
shared or not, all of them in one slice of the tokens and in several; at sizes whose tiles, stages and pieces end anywhere.

Bound, as everywhere for this operator: fp32 additions of `tokens` exact products in any order, two operations behind them, and half a step where C is bf16."""
import pytest

import test_gpu_training_ops as small

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ah = small.ah

SIZES = [  # tokens, d_out, d_in; tile, shares of the tokens in a workgroup, whether there are several slices
    (1001, 2056, 4104, 256, 1, False), (300, 5000, 3001, 256, 1, False), (31, 2056, 4104, 256, 1, False), (1, 5102, 1552, 256, 1, False), (0, 2056, 4104, 256, 1, False),
    (12617, 4091, 2045, 256, 1, True), (4097, 2300, 2300, 256, 1, True), (20001, 1500, 1499, 256, 1, True),
    (33, 4100, 4104, 128, 1, False), (1001, 4099, 4103, 128, 1, False), (2049, 2203, 2199, 128, 1, False), (1, 4100, 4104, 128, 1, False), (0, 4100, 4104, 128, 1, False),
    (2278, 21, 5524, 128, 1, True),
    (1001, 2047, 2048, 128, 2, False), (4097, 2000, 999, 128, 2, True),
]


def product(G, x):
    """G^T x in 64 bits"""
    return torch.matmul(G.t().contiguous(), x)


def operands(ah, tokens, d_out, d_in, gap):
    """G with NaN between its rows, and a checkpoint with codes of NaN between its."""
    gen = torch.Generator(device="cuda").manual_seed(tokens * 3 + d_out + d_in)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    G = torch.full((max(tokens, 1), (d_out + 7) // 8 * 8 + gap), float("nan"), dtype=torch.bfloat16, device="cuda")[:tokens, :d_out]
    G.copy_(r(tokens, d_out).mul_(1e-3))
    x = r(tokens, d_in) * torch.exp2(torch.randint(-4, 5, (tokens, 1), generator=gen, device="cuda").float())
    codes = torch.full((tokens, (d_in + 15) // 16 * 16 + 2 * gap), 127, dtype=torch.uint8, device="cuda")[:, :d_in]
    x8 = (codes, torch.empty(tokens, (d_in + 31) // 32, dtype=torch.uint8, device="cuda"))
    ah.adahop_ckpt8_pack(x, out=x8)
    return gen, G, x8, G.double(), ah.adahop_ckpt8_unpack(x8, dtype=torch.float32).double()


def check_plan(ah, tokens, d_out, d_in, tile, shares, sliced):
    got = ah.adahop_debug_ckpt8_wgrad_plan(tokens, d_out, d_in)
    assert got[:2] == (tile, shares) and (got[2] > 1) == sliced, f"another kernel than this test is of: {got}"


@pytest.mark.parametrize("tokens,d_out,d_in,tile,shares,sliced", SIZES)
def test_against_64_bits(ah, tokens, d_out, d_in, tile, shares, sliced):
    check_plan(ah, tokens, d_out, d_in, tile, shares, sliced)
    gen, G, x8, G64, x64 = operands(ah, tokens, d_out, d_in, 0 if tokens % 2 else 8)
    C64, mag = product(G64, x64), product(G64.abs(), x64.abs())
    eps = 2.0 ** -24
    for scaled, add, bf16_out, pad in ((False, False, False, 0), (True, True, False, 3), (True, False, True, 1), (False, True, True, 0)):
        dtype = torch.bfloat16 if bf16_out else torch.float32
        scale = torch.randn(d_in, generator=gen, device="cuda").mul_(0.2).add_(1.0).to(torch.bfloat16 if add else torch.float32) if scaled else None
        more = torch.randn(d_out, d_in, generator=gen, device="cuda").mul_(1e-2).to(dtype) if add else None
        room = torch.full((d_out, d_in + pad), 7.0, dtype=dtype, device="cuda")
        small.say("wgrad kernels", tokens, d_out, d_in, scaled, add, bf16_out)
        ah.adahop_ckpt8_wgrad(G, x8, col_scale=scale, add=more, Cout=room[:, :d_in])
        want, m = (C64, mag) if scale is None else (C64 * scale.double(), mag * scale.double().abs())
        bound = (2 * tokens + 16) * eps * m + 1e-37
        if add:
            want = want + more.double()
            bound += 2 * eps * (want.abs() + more.double().abs())
        if bf16_out:
            bound += small.BF16 * want.abs()
        over = ((room[:, :d_in].double() - want).abs() / bound).max().item()
        assert over <= 1.0, f"{over:.2f} times what is allowed"
        assert bool((room[:, d_in:] == 7.0).all())
        again = ah.adahop_ckpt8_wgrad(G, x8, col_scale=scale, add=more, Cout=more)     # on top of what is there, or somewhere new
        assert torch.equal(again if add or not bf16_out else again.to(dtype), room[:, :d_in]), "other bits in a second call"


@pytest.mark.parametrize("tokens,d_out,d_in,tile,shares,sliced", [s for s in SIZES if s[0] > 1])
def test_infinities_and_nan_stay_in_their_sums(ah, tokens, d_out, d_in, tile, shares, sliced):
    """In the last token, behind which a stage ends in rows that are not there, and in the first."""
    check_plan(ah, tokens, d_out, d_in, tile, shares, sliced)
    _, G, x8, _, _ = operands(ah, tokens, d_out, d_in, 8)
    clean = ah.adahop_ckpt8_wgrad(G, x8)
    rows, cols = (d_out - 1, d_out // 3), (d_in - 1, d_in // 3)
    G[tokens - 1, rows[0]], G[0, rows[1]] = float("inf"), float("nan")
    x8[0][tokens - 1, cols[0]], x8[0][0, cols[1]] = 127, 255
    small.say("infinities in wgrad kernels", tokens, d_out, d_in)
    got = ah.adahop_ckpt8_wgrad(G, x8)
    assert not any(bool(got[r].isfinite().any()) for r in rows) and all(bool(got[:, c].isnan().all()) for c in cols)
    rest = torch.ones_like(got, dtype=torch.bool)
    rest[list(rows)], rest[:, list(cols)] = False, False
    assert torch.equal(got[rest], clean[rest])
