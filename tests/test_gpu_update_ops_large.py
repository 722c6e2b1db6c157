"""The loss over a vocabulary and the updates at sizes where offsets pass 32 bits, the vocabulary comes in pieces or tiles in rounds, against products of torch in wider types."""
import pytest

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


def operands(T, D, V, ignored=0.1, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn(T, D, generator=g, device="cuda").to(torch.bfloat16)
    w = torch.empty(V, D, dtype=torch.bfloat16, device="cuda")
    for i in range(0, V, 1 << 16):
        w[i:i + (1 << 16)] = torch.randn(min(1 << 16, V - i), D, generator=g, device="cuda") * D ** -0.5
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    return h, w, torch.where(torch.rand(T, generator=g, device="cuda") < ignored, -100, y)


def lse_of(h, w, at_once):
    parts = [torch.logsumexp(h.double() @ w[i:i + at_once].double().t(), 1) for i in range(0, w.shape[0], at_once)]
    return torch.logsumexp(torch.stack(parts), 0)


# tokens, dim, vocabulary: whole rounds of large tiles with a rest in small ones; large tiles alone; a wide row for few tokens; few tokens, a vocabulary whose far rows pass 2^31 elements
@pytest.mark.parametrize("T,D,V", [(600, 1024, 30000), (2100, 256, 9000), (4, 8200, 3000), (8, 8200, 3000), (3, 2056, 1050001)])
def test_loss(ah, T, D, V):
    say("loss", T, D, V)
    h, w, y = operands(T, D, V)
    y[0] = V - 1
    out = ah.adahop_linear_ce(h, w, y)
    want = lse_of(h, w, 1 << 15)
    # a logit is a sum of D products of which each is off by roundings of the sum so far; here |z| < 8 and sum |h w| < D / 4 at these sizes
    bound = (D / 4 + 16) * U32 * D ** 0.5 + 200 * U32
    assert ((out["lse"].double() - want).abs() <= bound).all()
    at = (h.double() * w[y.clamp(min=0)].double()).sum(1)
    loss = torch.where(y >= 0, want - at, torch.zeros_like(want))
    assert ((out["loss"].double() - loss).abs() <= 2 * bound).all()


# pieces of the vocabulary (more than 2^29 logits); d_w past 2^31 elements
@pytest.mark.parametrize("T,D,V", [(8200, 72, 66001), (3, 2056, 1050001)])
def test_gradients(ah, T, D, V):
    say("gradients", T, D, V)
    h, w, y = operands(T, D, V)
    y[0] = V - 1
    lse = ah.adahop_linear_ce(h, w, y)["lse"]
    g = torch.rand(T, device="cuda") + 0.5
    out = ah.adahop_linear_ce_backward(h, w, y, lse, g, d_w_bf16=True)
    want_h, size_h = (torch.zeros(T, D, dtype=torch.float64, device="cuda") for _ in range(2))
    there = (y >= 0).double()[:, None]
    for i in range(0, V, 1 << 14):
        part = w[i:i + (1 << 14)].double()
        dz = torch.exp(h.double() @ part.t() - lse.double()[:, None])
        rows = torch.nonzero((y >= i) & (y < i + part.shape[0]))[:, 0]
        dz[rows, y[rows] - i] -= 1.0
        dz *= there * g.double()[:, None]
        want_h += dz @ part
        size_h += dz.abs() @ part.abs()
        if i == 0 or i + (1 << 14) >= V or i // (1 << 14) == 40:        # the first words, the last ones, some between
            want = dz.t() @ h.double()
            # dz rounded to bf16 and its exponential's error, by the other operand; then the result's own rounding
            bound = (BF16 + 64 * U32) * (dz.abs().t() @ h.double().abs()) * 1.01 + BF16 * want.abs() + 1e-30
            assert ((out["d_w"][i:i + part.shape[0]].double() - want).abs() <= bound).all(), i
    bound = (BF16 + (V / 4 + 64) * U32) * size_h * 1.01 + BF16 * want_h.abs() + 1e-30
    assert ((out["d_h"].double() - want_h).abs() <= bound).all()
    assert not out["d_h"][y < 0].any()


def test_orthogonalize_one_step_of_a_large_matrix(ah):
    """65536 x 16384, 2^30 elements: out v = a X v + b X (X^T X v) + c X (X^T X)^2 v for a few vectors v, of which each product is formed in 64 bits."""
    say("orthogonalize 65536 x 16384")
    rows, cols, (a, b, c) = 65536, 16384, (3.4445, -4.7750, 2.0315)
    gen = torch.Generator(device="cuda").manual_seed(1)
    g = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    strong = [torch.randn(n, 4, generator=gen, device="cuda") for n in (rows, cols)]
    for i in range(0, rows, 4096):
        g[i:i + 4096] = torch.randn(4096, cols, generator=gen, device="cuda") + 4.0 * strong[0][i:i + 4096] @ strong[1].t()
    out = ah.adahop_orthogonalize(g, steps=1)

    def times(m, v):
        return torch.cat([m[i:i + 4096].double() @ v for i in range(0, rows, 4096)])

    def turned(m, v):
        return sum(m[i:i + 4096].double().t() @ v[i:i + 4096] for i in range(0, rows, 4096))
    norm = sum(g[i:i + 4096].double().square().sum() for i in range(0, rows, 4096)).sqrt()
    v = torch.cat((strong[1].double()[:, :2], torch.randn(cols, 2, generator=gen, device="cuda", dtype=torch.float64)), 1)
    x = times(g, v) / norm
    gram = lambda u: turned(g, times(g, u) / norm) / norm  # noqa: E731
    once = gram(v)
    twice = gram(once)
    want = a * x + (b * times(g, once) + c * times(g, twice)) / norm
    got = times(out, v)
    # per vector: the roundings to fp16 and bf16 (2^-11, 2^-8) are independent over elements and average along it
    off = (got - want).norm(dim=0) / want.norm(dim=0)
    assert (off < 2 * BF16).all(), off


def test_update_of_a_tall_matrix_with_rounds_of_tiles(ah):
    """9000 x 2050: several rounds of tiles with a rest in slices, sides that end inside them; against the same iteration in 64 bits on the GPU."""
    say("update 9000 x 2050")
    gen = torch.Generator(device="cuda").manual_seed(2)
    for m, n in ((9000, 2050), (2050, 9000)):
        w, g, mom = (torch.randn(m, n, generator=gen, device="cuda") * s for s in (0.02, 1.0, 3.0))
        was = [t.double() for t in (w, g, mom)]
        ah.adahop_muon_update(w, g, mom, 0.05, scale=0.5)
        m1 = 0.95 * was[2] + was[1]
        u = was[1] + 0.95 * m1
        x = u / (u.norm() + 1e-7)
        for _ in range(5):
            gram = x @ x.t() if m <= n else x.t() @ x
            p = -4.7750 * gram + 2.0315 * gram @ gram
            x = 3.4445 * x + (p @ x if m <= n else x @ p)
        step = 0.05 * 0.5 * x
        assert (mom.double() - m1).abs().max() <= 4 * U32 * (m1.abs().max() + was[1].abs().max())
        # at a smaller side of 2050 the roundings to fp16 make some 3e-4 of the result (newton_schulz_held); three times that
        off = (w.double() - (was[0] - step)).norm()
        assert off <= 1e-3 * step.norm() + 2 * U32 * was[0].norm(), (off / step.norm()).item()
