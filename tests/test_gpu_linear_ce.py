"""The loss over a vocabulary and its gradients on the GPU against their 64-bit definitions (oracle/update.py).

Bounds.  A logit is a sum of dim products of bf16 numbers (exact in fp32) by dim / 32 matrix instructions; each is taken to be off by at most 8 roundings of
2^-24 of the magnitude m = sum |h w| it sums up (32 additions in a tree, with truncation): EZ = (dim / 4 + 16) 2^-24 |logit_scale| m.  lse is off by at most the largest
such error of the row, by the relative error of a sum of exponentials (each 2^-23 times its argument, and at most 128 additions in a row) and by its own
rounding.  dz is off by its rounding to bf16, 2^-8, and the errors of its exponential; a gradient by these times the other operand, and by its fp32 sum and
rounding."""
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


def bf16(a):
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16).double().numpy()


def up(a, dtype=torch.bfloat16, pad=0, offset=0):
    """A numpy array as a GPU tensor, rows `pad` elements further apart than they are long, beginning `offset` elements into memory full of NaN."""
    t = torch.from_numpy(np.ascontiguousarray(a)).to(dtype)
    room = torch.full((t.shape[0] * (t.shape[1] + pad) + offset,), float("nan"), dtype=dtype, device="cuda")
    v = room[offset:].view(t.shape[0], t.shape[1] + pad)[:, :t.shape[1]]
    v.copy_(t)
    return v


def down(t):
    return t.detach().double().cpu().numpy()


class Case:
    def __init__(self, T, D, V, seed=0, ignored=0.2, logit_scale=1.0, z_loss=0.0, spread=1.0):
        r = np.random.default_rng([seed, T, D, V])
        self.h, self.w = bf16(r.normal(size=(T, D))), bf16(r.normal(size=(V, D)) * spread * D ** -0.5)
        self.targets = np.where(r.random(T) < ignored, -100, r.integers(0, V, T))
        self.d_loss = r.normal(size=T).astype(np.float32).astype(np.float64)
        self.options = dict(logit_scale=logit_scale, z_loss=z_loss)
        self.loss, self.lse = orc.linear_ce(self.h, self.w, self.targets, **self.options)
        self.lse32 = self.lse.astype(np.float32).astype(np.float64)
        self.ez = ((D / 4 + 16) * U32 * abs(logit_scale) * (np.abs(self.h) @ np.abs(self.w).T))
        z = np.abs(orc.logits(self.h, self.w, logit_scale) - self.lse[:, None])
        self.e_exp = self.ez + 2 * U32 * z + 8 * U32            # relative error of exp(z - lse), as long as it matters

    def check_forward(self, out, what=""):
        e_lse = self.ez.max(axis=1) + 160 * U32 + 2 * U32 * np.abs(self.lse)
        off = np.abs(down(out["lse"]) - self.lse)
        assert np.all(off <= e_lse), (what, off.max(), e_lse.min())
        z_loss = abs(self.options["z_loss"])
        e_loss = e_lse + self.ez.max(axis=1) + 2 * z_loss * np.abs(self.lse) * e_lse + 4 * U32 * (np.abs(self.loss) + np.abs(self.lse) + z_loss * self.lse ** 2)
        off = np.abs(down(out["loss"]) - self.loss)
        assert np.all(off <= e_loss), (what, off.max(), e_loss.min())
        assert np.all(down(out["loss"])[self.targets < 0] == 0)

    def gradients(self, dh, dw, add=0.0, what=""):
        """dh, dw: (tensor, whether it is fp32) or None"""
        dz = orc.linear_ce_dz(self.h, self.w, self.targets, self.lse32, self.d_loss, **self.options)
        gain = np.where(self.targets >= 0, np.abs(self.d_loss * self.options["logit_scale"]), 0.0)[:, None]
        p = np.exp(orc.logits(self.h, self.w, self.options["logit_scale"]) - self.lse32[:, None]) * np.abs(1 + 2 * self.options["z_loss"] * self.lse32)[:, None]
        e_dz = BF16 * np.abs(dz) + (self.e_exp + 8 * U32) * p * gain * (1 + BF16)
        for given, want, err, n in ((dh, dz @ self.w, (e_dz @ np.abs(self.w), np.abs(dz) @ np.abs(self.w)), self.w.shape[0]),
                                    (dw, dz.T @ self.h + add, (e_dz.T @ np.abs(self.h), np.abs(dz).T @ np.abs(self.h)), self.h.shape[0])):
            if given is None:
                continue
            got, f32 = given
            bound = err[0] + (n / 4 + 16) * U32 * err[1] + 2 * U32 * np.abs(want)
            bound = bound + (0.0 if f32 else BF16 * (np.abs(want) + bound)) + 1e-37
            off = np.abs(down(got) - want)
            assert np.all(off <= bound), (what, n, (off / bound).max())


SIZES = [(1, 8, 1), (1, 64, 300), (2, 1032, 9000), (3, 40, 257), (5, 504, 1003), (8, 512, 34), (8, 4104, 2051), (9, 512, 64), (16, 128, 1000), (17, 72, 129), (127, 96, 255), (130, 264, 513), (257, 33, 1001), (300, 1024, 700), (520, 64, 2050)]


@pytest.mark.parametrize("T,D,V", SIZES)
def test_loss(ah, T, D, V):
    say("loss", T, D, V)
    c = Case(T, D, V, z_loss=1e-3, logit_scale=0.7)
    out = ah.adahop_linear_ce(up(c.h), up(c.w), torch.from_numpy(c.targets).cuda(), **c.options)
    torch.cuda.synchronize()
    c.check_forward(out)


@pytest.mark.parametrize("T,D,V", SIZES)
def test_gradients(ah, T, D, V):
    say("gradients", T, D, V)
    c = Case(T, D, V, z_loss=1e-3, logit_scale=0.7)
    h, w, t = up(c.h), up(c.w), torch.from_numpy(c.targets).cuda()
    lse, g = torch.from_numpy(c.lse32).float().cuda(), torch.from_numpy(c.d_loss).float().cuda()
    for d_w_bf16 in (False, True):
        out = ah.adahop_linear_ce_backward(h, w, t, lse, g, d_w_bf16=d_w_bf16, **c.options)
        torch.cuda.synchronize()
        assert out["d_h"].dtype == torch.bfloat16 and out["d_w"].dtype == (torch.bfloat16 if d_w_bf16 else torch.float32)
        c.gradients((out["d_h"], False), (out["d_w"], not d_w_bf16))


@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 0), (0, 1), (5, 3)])
@pytest.mark.parametrize("T,D,V", [(70, 96, 300), (33, 41, 131)])
def test_strides_and_alignments(ah, T, D, V, pad, offset):
    """Rows further apart than they are long, with NaN between them, on and off the alignments that are read in place."""
    say("strides", T, D, V, pad, offset)
    c = Case(T, D, V)
    h, w, t = up(c.h, pad=pad, offset=offset), up(c.w, pad=pad, offset=offset), torch.from_numpy(c.targets).cuda()
    c.check_forward(ah.adahop_linear_ce(h, w, t))
    room = {"d_h": torch.full((T, D + pad), 7, dtype=torch.bfloat16, device="cuda"), "d_w": torch.full((V, D + pad), 7, dtype=torch.float32, device="cuda")}
    out = ah.adahop_linear_ce_backward(h, w, t, torch.from_numpy(c.lse32).float().cuda(), torch.from_numpy(c.d_loss).float().cuda(),
                                       **{k: v[:, :D] for k, v in room.items()})
    torch.cuda.synchronize()
    c.gradients((out["d_h"], False), (out["d_w"], True))
    assert all(bool((v[:, D:] == 7).all()) for v in room.values())


def test_added_to_and_one_of_the_two(ah):
    say("added to")
    c = Case(200, 64, 400)
    h, w, t = up(c.h), up(c.w), torch.from_numpy(c.targets).cuda()
    lse, g = torch.from_numpy(c.lse32).float().cuda(), torch.from_numpy(c.d_loss).float().cuda()
    before = np.random.default_rng(3).normal(size=(400, 64)).astype(np.float32)
    d_w = torch.from_numpy(before).cuda()
    out = ah.adahop_linear_ce_backward(h, w, t, lse, g, d_w=d_w, add=d_w, want_h=False)
    assert out["d_h"] is None and out["d_w"] is d_w
    c.gradients(None, (d_w, True), add=before.astype(np.float64))
    out = ah.adahop_linear_ce_backward(h, w, t, lse, g, want_w=False)
    assert out["d_w"] is None
    c.gradients((out["d_h"], False), None)


def test_one_gradient_for_all_tokens(ah):
    """d_loss expanded from one number, and none at all."""
    say("d_loss")
    c = Case(90, 64, 400)
    h, w, t, lse = up(c.h), up(c.w), torch.from_numpy(c.targets).cuda(), torch.from_numpy(c.lse32).float().cuda()
    for d_loss, value in ((torch.full((1,), 0.25, device="cuda").expand(90), 0.25), (None, 1.0)):
        c.d_loss = np.full(90, value)
        out = ah.adahop_linear_ce_backward(h, w, t, lse, d_loss)
        torch.cuda.synchronize()
        c.gradients((out["d_h"], False), (out["d_w"], True))


def test_no_token_has_a_target(ah):
    say("no targets")
    c = Case(50, 64, 200, ignored=2.0)
    h, w, t = up(c.h), up(c.w), torch.from_numpy(c.targets).cuda()
    out = ah.adahop_linear_ce(h, w, t)
    assert not out["loss"].any()
    back = ah.adahop_linear_ce_backward(h, w, t, out["lse"])
    assert not back["d_h"].any() and not back["d_w"].any()


def test_no_tokens(ah):
    say("no tokens")
    w = torch.randn(200, 64, device="cuda").to(torch.bfloat16)
    h, t = w[:0], torch.zeros(0, dtype=torch.int64, device="cuda")
    assert ah.adahop_linear_ce(h, w, t)["loss"].shape == (0,)
    lse = torch.zeros(0, device="cuda")
    assert not ah.adahop_linear_ce_backward(h, w, t, lse)["d_w"].any()
    add = torch.randn(200, 64, device="cuda")
    assert torch.equal(ah.adahop_linear_ce_backward(h, w, t, lse, add=add)["d_w"], add)


def test_tokens_without_a_target_take_no_part_whatever_they_hold(ah):
    """Padding holds infinities and NaN: the other tokens' gradients are as without it."""
    say("padding")
    c = Case(300, 64, 500, ignored=0.3)
    h, w, t = up(c.h), up(c.w), torch.from_numpy(c.targets).cuda()
    g = torch.from_numpy(c.d_loss).float().cuda()
    lse = torch.from_numpy(c.lse32).float().cuda()
    want = ah.adahop_linear_ce_backward(h, w, t, lse, g)
    masked = torch.nonzero(t < 0)[:, 0]
    h, lse, g = h.clone(), lse.clone(), g.clone()
    for k, v in enumerate((float("nan"), float("inf"), -3e38)):
        h[masked[k::3]] = v
    lse[masked], g[masked] = float("nan"), float("inf")
    got = ah.adahop_linear_ce_backward(h, w, t, lse, g)
    torch.cuda.synchronize()
    assert torch.equal(got["d_h"], want["d_h"]) and torch.equal(got["d_w"], want["d_w"])
    f = ah.adahop_linear_ce(h, w, t)
    there = t >= 0
    assert not f["loss"][~there].any() and torch.equal(f["loss"][there], ah.adahop_linear_ce(up(c.h), w, t)["loss"][there])


def test_a_target_outside_the_vocabulary_is_seen(ah):
    say("target outside")
    c = Case(40, 64, 100, ignored=0.0)
    t = torch.from_numpy(c.targets).cuda()
    t[7] = 100
    out = ah.adahop_linear_ce(up(c.h), up(c.w), t)
    assert torch.isnan(out["loss"][7]) and torch.isfinite(out["lse"]).all() and int(torch.isnan(out["loss"]).sum()) == 1
    back = ah.adahop_linear_ce_backward(up(c.h), up(c.w), t, out["lse"])
    assert torch.isnan(back["d_h"][7]).all() and torch.isnan(back["d_w"]).all() and int(torch.isnan(back["d_h"]).any(1).sum()) == 1


def test_large_and_equal_logits(ah):
    """Logits far beyond the range of exp, and a row of equal ones."""
    say("large logits")
    c = Case(64, 64, 600, spread=200.0)
    h, w, t = up(c.h), up(c.w), torch.from_numpy(c.targets).cuda()
    out = ah.adahop_linear_ce(h, w, t)
    c.check_forward(out)
    h0 = torch.zeros_like(h)
    out = ah.adahop_linear_ce(h0, w, t)
    assert torch.allclose(out["lse"], torch.full_like(out["lse"], float(np.log(600.0))), rtol=4 * U32, atol=0)


def test_the_same_bits_in_every_call(ah):
    say("same bits")
    c = Case(700, 128, 3000)
    h, w, t = up(c.h), up(c.w), torch.from_numpy(c.targets).cuda()
    one = ah.adahop_linear_ce(h, w, t)
    b1 = ah.adahop_linear_ce_backward(h, w, t, one["lse"])
    for _ in range(3):
        two = ah.adahop_linear_ce(h, w, t)
        b2 = ah.adahop_linear_ce_backward(h, w, t, two["lse"])
        assert torch.equal(one["loss"], two["loss"]) and torch.equal(b1["d_h"], b2["d_h"]) and torch.equal(b1["d_w"], b2["d_w"])


def test_gradients_are_the_slopes(ah):
    """Differences of the loss itself, along random directions of h and w."""
    say("slopes")
    c = Case(48, 64, 300, ignored=0.1, z_loss=1e-2)
    h, w, t = up(c.h), up(c.w), torch.from_numpy(c.targets).cuda()
    lse = ah.adahop_linear_ce(h, w, t, **c.options)["lse"]
    out = ah.adahop_linear_ce_backward(h, w, t, lse, **c.options)
    r = np.random.default_rng(5)
    for name, x in (("d_h", c.h), ("d_w", c.w)):
        d = r.normal(size=x.shape)
        step = 1e-4
        at = [orc.linear_ce(*(c.h + s * d, c.w) if name == "d_h" else (c.h, c.w + s * d), c.targets, **c.options)[0].sum() for s in (step, -step)]
        slope, got = (at[0] - at[1]) / (2 * step), (down(out[name]) * d).sum()
        # each gradient element is off by at most 2^-8 of itself and 2^-8 of what it sums up; along a random direction such errors add as roots of squares
        size = np.sqrt((down(out[name]) ** 2).sum())
        assert abs(got - slope) <= 8 * 2 * BF16 * size, (name, got, slope, size)
