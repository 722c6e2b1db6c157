"""Orthogonalisation by Newton-Schulz products and the update of a weight on the GPU against their 64-bit definitions (oracle/update.py).

Bounds.  The result's distance from exact arithmetic is that of the roundings to fp16 on the way, which the steps amplify by an amount that depends on the
matrix.  The oracle makes the same roundings at the same places (newton_schulz_held); another order of the fp32 sums moves some of them to the other side of a
tie and is otherwise 2^13 times smaller than they are, so the distance is allowed to be twice the oracle's own, and the amplified fp32 sums' 64 * 2^-24 * the same
amplification (the oracle's distance over 2^-12) more.  bf16 results: half a step, 2^-8 of each value, more."""
import numpy as np
import pytest

from oracle import update as orc

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U32, BF16 = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def ah():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_02525_amd import binding
    binding.lib()
    return binding


def say(*a):
    print("[case]", *a, flush=True)


def down(t):
    return t.detach().double().cpu().numpy()


def matrix(kind, m, n, seed=0):
    r = np.random.default_rng([seed, m, n])
    g = r.normal(size=(m, n))
    if kind == "strong":        # a few strong directions
        g = 0.02 * g + r.normal(size=(m, 8)) @ r.normal(size=(8, n))
    elif kind == "one":         # one direction alone
        g = r.normal(size=(m, 1)) @ r.normal(size=(1, n))
    elif kind == "rows":        # a few rows far larger than the others
        g[: max(1, m // 200)] *= 100.0
    elif kind == "empty":       # rows and columns of zeros
        g[m // 3:m // 2] = 0.0
        g[:, n // 4:n // 3] = 0.0
    return g


def up(a, f32=False, pad=0, offset=0):
    dtype = torch.float32 if f32 else torch.bfloat16
    t = torch.from_numpy(np.ascontiguousarray(a)).to(dtype)
    room = torch.full((t.shape[0] * (t.shape[1] + pad) + offset,), float("nan"), dtype=dtype, device="cuda")
    v = room[offset:].view(t.shape[0], t.shape[1] + pad)[:, :t.shape[1]]
    v.copy_(t)
    return v


def distance(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


def bound(u, want, **how):
    """Of the distance of an fp32 result."""
    own = distance(orc.newton_schulz_held(u, split=min(u.shape) <= 128, **how), want)
    return 2.0 * own + 64 * U32 * own * 2.0 ** 12 + 64 * U32


SIZES = [(1, 1), (1, 70), (70, 1), (2, 3), (31, 33), (64, 64), (48, 600), (600, 48), (129, 255), (256, 256), (257, 300), (300, 257), (520, 1030), (1030, 520)]


@pytest.mark.parametrize("m,n", SIZES)
@pytest.mark.parametrize("kind", ["plain", "strong"])
def test_orthogonalize(ah, m, n, kind):
    say("orthogonalize", m, n, kind)
    g = up(matrix(kind, m, n))
    u = down(g)
    want = orc.newton_schulz(u)
    most = bound(u, want)
    for dtype, more in ((torch.float32, 0.0), (torch.bfloat16, BF16)):
        out = ah.adahop_orthogonalize(g, dtype=dtype)
        torch.cuda.synchronize()
        assert out.dtype == dtype and out.shape == (m, n)
        assert distance(down(out), want) <= most + more, (distance(down(out), want), most)


@pytest.mark.parametrize("kind", ["one", "rows", "empty"])
@pytest.mark.parametrize("m,n", [(96, 200), (400, 300)])
def test_matrices_of_other_kinds(ah, m, n, kind):
    say("kinds", m, n, kind)
    g = up(matrix(kind, m, n), f32=True)
    u = down(g)
    want = orc.newton_schulz(u)
    out = ah.adahop_orthogonalize(g, dtype=torch.float32)
    assert distance(down(out), want) <= bound(u, want)
    if kind == "empty":
        assert not out[m // 3:m // 2].any() and not out[:, n // 4:n // 3].any()


@pytest.mark.parametrize("steps,coefficients", [(1, (3.4445, -4.7750, 2.0315)), (2, (3.4445, -4.7750, 2.0315)), (6, (1.875, -1.25, 0.375)), (12, (1.5, -0.5, 0.0))])
def test_steps_and_coefficients(ah, steps, coefficients):
    say("steps", steps, coefficients)
    g = up(matrix("plain", 270, 330), f32=True)
    u = down(g)
    how = dict(steps=steps, coefficients=coefficients)
    want = orc.newton_schulz(u, **how)
    out = ah.adahop_orthogonalize(g, dtype=torch.float32, scale=2.5, **how)
    assert distance(down(out), 2.5 * want) <= bound(u, want, **how)


@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 1), (1, 0)])
@pytest.mark.parametrize("m,n", [(100, 140), (300, 270)])
def test_strides_and_alignments(ah, m, n, pad, offset):
    say("strides", m, n, pad, offset)
    a = matrix("plain", m, n)
    g = up(a, pad=pad, offset=offset)
    room = torch.full((m, n + pad), 7, dtype=torch.bfloat16, device="cuda")
    ah.adahop_orthogonalize(g, out=room[:, :n])
    want = ah.adahop_orthogonalize(up(a))
    torch.cuda.synchronize()
    assert torch.equal(room[:, :n], want) and bool((room[:, n:] == 7).all())


@pytest.mark.parametrize("size", [1e-30, 1e30])
def test_very_small_and_very_large_elements(ah, size):
    """Squares beyond the range of fp32."""
    say("size", size)
    g = up(matrix("plain", 140, 270) * size, f32=True)
    u = down(g)
    want = orc.newton_schulz(u, eps=0.0)
    assert distance(down(ah.adahop_orthogonalize(g, dtype=torch.float32, eps=0.0)), want) <= bound(u, want, eps=0.0)


def test_zero_and_not_finite(ah):
    say("zero")
    g = torch.zeros(140, 270, device="cuda")
    assert not ah.adahop_orthogonalize(g).any()
    for v in (float("nan"), float("inf"), float("-inf")):
        g = torch.ones(140, 270, device="cuda")
        g[3, 5] = v
        assert torch.isnan(ah.adahop_orthogonalize(g)).all()


def weights(m, n, seed=7):
    r = np.random.default_rng([seed, m, n])
    return [r.normal(size=(m, n)) * s for s in (0.02, 1.0, 3.0)]


def check_update(out, w, g, m0, rate, mu, decay, nesterov, scale, w32=True):
    """w, g, m0: as the GPU got them, in 64 bits"""
    m, u = orc.momentum(m0, g, mu, nesterov)
    assert np.all(np.abs(down(out["momentum"]) - m) <= 4 * U32 * (np.abs(mu * m0) + np.abs(g)))
    x = orc.newton_schulz(u)
    off = down(out["w"]) - ((1 - rate * decay) * w - rate * scale * x)
    own = bound(u, x) * rate * scale * np.linalg.norm(x)
    assert np.linalg.norm(off) <= own + (4 * U32 if w32 else BF16) * (np.linalg.norm(w) * (1 + rate * decay) + rate * scale * np.linalg.norm(x))


@pytest.mark.parametrize("m,n", [(1, 1), (40, 30), (200, 330), (330, 200), (700, 300)])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("f32", [True, False])
def test_update(ah, m, n, nesterov, f32):
    say("update", m, n, nesterov, f32)
    w0, g0, m0 = weights(m, n)
    w, g, mom = up(w0, True), up(g0, f32), up(m0, True)
    was = [down(t) for t in (w, g, mom)]
    copy = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    out = ah.adahop_muon_update(w, g, mom, 0.02, mu=0.9, weight_decay=0.1, nesterov=nesterov, w_bf16=copy)
    torch.cuda.synchronize()
    assert out["w"] is w and out["momentum"] is mom and out["w_bf16"] is copy
    assert torch.equal(copy, w.to(torch.bfloat16))
    check_update(out, *was, 0.02, 0.9, 0.1, nesterov, max(1.0, m / n) ** 0.5)


def test_update_beside_and_in_bf16(ah):
    """Outputs of their own leave the inputs as they are, and hold the same bits as in place; weights in bf16."""
    say("update beside")
    w0, g0, m0 = weights(300, 270)
    for f32 in (True, False):
        w, g, mom = up(w0, f32, pad=3), up(g0, pad=1), up(m0, True, pad=2)
        was = [t.clone() for t in (w, g, mom)]
        out = ah.adahop_muon_update(w, g, mom, 0.02, scale=0.3, w_out=torch.empty_like(was[0]), momentum_out=torch.empty_like(was[2]))
        assert all(torch.equal(a, b) for a, b in zip((w, g, mom), was))
        check_update(out, *(down(t) for t in was), 0.02, 0.95, 0.0, True, 0.3, w32=f32)
        ah.adahop_muon_update(w, g, mom, 0.02, scale=0.3)
        assert torch.equal(w, out["w"]) and torch.equal(mom, out["momentum"])


def test_the_same_bits_in_every_call(ah):
    say("same bits")
    for m, n in ((200, 3000), (600, 520), (2000, 300)):
        g = up(matrix("strong", m, n))
        one = ah.adahop_orthogonalize(g)
        for _ in range(3):
            assert torch.equal(one, ah.adahop_orthogonalize(g))
