"""The loss over a vocabulary and the updates by Newton-Schulz products: their definitions against differences, and what the entry points and the binding refuse (no GPU)."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import update as orc  # noqa: E402
from paper_2604_02525_amd import binding as ah  # noqa: E402

BAD, SPACE = ah.ADAHOP_E_INVALID_ARG, ah.ADAHOP_E_WORKSPACE
FAKE = 0x10000  # never dereferenced: every call here is refused


def test_gradients_of_the_loss_are_the_slopes():
    r = np.random.default_rng(0)
    h, w, targets, g = r.normal(size=(7, 5)), r.normal(size=(11, 5)), np.array([0, 10, -1, 3, 3, -100, 5]), r.normal(size=7)
    how = dict(logit_scale=0.6, z_loss=0.05)
    d_h, d_w = orc.linear_ce_backward(h, w, targets, orc.linear_ce(h, w, targets, **how)[1], g, **how)
    for x, d in ((h, d_h), (w, d_w)):
        for i in np.ndindex(x.shape):
            was, at = x[i], []
            for s in (1e-5, -1e-5):
                x[i] = was + s
                at.append((orc.linear_ce(h, w, targets, **how)[0] * g).sum())
            x[i] = was
            assert abs((at[0] - at[1]) / 2e-5 - d[i]) < 1e-8


def test_newton_schulz_moves_singular_values_alone():
    r = np.random.default_rng(1)
    for shape in ((6, 9), (9, 6), (5, 5)):
        g = r.normal(size=shape)
        u, s, vt = np.linalg.svd(g, full_matrices=False)
        s = s / (np.sqrt((g * g).sum()) + 1e-7)
        a, b, c = orc.NEWTON_SCHULZ
        for _ in range(5):
            s = a * s + b * s ** 3 + c * s ** 5
        assert np.allclose(orc.newton_schulz(g), (u * s) @ vt, atol=1e-12)
        held = orc.newton_schulz_held(g)
        assert np.linalg.norm(held - orc.newton_schulz(g)) < 0.02 * np.linalg.norm(held)


def t(data=FAKE, ld=64, f32=0):
    return ah.adahop_tensor_t(data, ld, f32)


def loss(T=32, V=128, D=64, backward=False, ws=FAKE, size=1 << 40, stream=None, **more):
    p = ah.adahop_linear_ce_t(tokens=T, vocab=V, dim=D, h=t(), w=t(), targets=FAKE, logit_scale=1.0, z_loss=0.0, loss=FAKE, lse=FAKE, d_loss=FAKE, d_loss_stride=1,
                              d_h=t(), d_w=t())
    for k, v in more.items():
        setattr(p, k, v)
    f = ah.lib().adahop_linear_ce_backward if backward else ah.lib().adahop_linear_ce
    return f(C.byref(p), ws, size, stream)


def test_loss_refuses():
    for backward in (False, True):
        f = lambda **k: loss(backward=backward, **k)  # noqa: E731
        assert f(T=-1) == f(T=(1 << 21) + 1) == f(V=0) == f(D=0) == f(V=(1 << 21) + 1) == f(T=1 << 20, V=1 << 20) == f(V=1 << 20, D=1 << 16) == BAD
        assert f(h=t(data=None)) == f(w=t(data=None)) == f(targets=None) == f(targets=FAKE + 4) == BAD
        assert f(h=t(f32=1)) == f(w=t(f32=1)) == f(h=t(ld=63)) == f(w=t(ld=1 << 22)) == f(h=t(data=FAKE + 1)) == BAD
        assert f(logit_scale=float("inf")) == f(z_loss=float("nan")) == BAD
        assert f(ws=None) == f(ws=FAKE + 64) == f(size=100) == SPACE
    assert loss(loss=None, lse=None) == loss(loss=FAKE + 2) == loss(lse=FAKE + 1) == BAD
    b = lambda **k: loss(backward=True, **k)  # noqa: E731
    assert b(lse=None) == b(lse=FAKE + 2) == b(d_loss=FAKE + 1) == b(d_loss_stride=-1) == b(d_h=t(data=None), d_w=t(data=None)) == BAD
    assert b(d_h=t(ld=63)) == b(d_w=t(ld=8)) == b(d_w=t(f32=2)) == b(d_w=t(data=FAKE + 2, f32=1)) == b(add=t(ld=1)) == b(d_w=t(data=None), add=t()) == BAD
    L = ah.lib()
    assert L.adahop_linear_ce(None, FAKE, 1 << 40, None) == L.adahop_linear_ce_backward(None, FAKE, 1 << 40, None) == BAD
    assert L.adahop_linear_ce_workspace_bytes(None, 0) == 0


def ns(rows=64, cols=96, steps=5, a=3.0, b=-4.0, c=2.0, eps=1e-7, scale=1.0, g=t(ld=96), out=t(ld=96), ws=FAKE, size=1 << 40):
    m = ah.adahop_newton_schulz_t(rows, cols, steps, a, b, c, eps, scale)
    return ah.lib().adahop_orthogonalize(C.byref(m), g and C.byref(g), out and C.byref(out), ws, size, None)


def muon(rows=64, cols=96, method_rows=64, ws=FAKE, size=1 << 40, **more):
    m = ah.adahop_newton_schulz_t(method_rows, 96, 5, 3.0, -4.0, 2.0, 1e-7, 1.0)
    w32 = t(ld=96, f32=1)
    p = ah.adahop_muon_t(rows=rows, cols=cols, g=t(ld=96), momentum=w32, momentum_out=w32, w=w32, w_out=w32, w_bf16=t(ld=96), rate=0.1, mu=0.9, weight_decay=0.1, nesterov=1)
    for k, v in more.items():
        setattr(p, k, v)
    return ah.lib().adahop_muon_update(C.byref(m), C.byref(p), ws, size, None)


def test_newton_schulz_refuses():
    assert ns(rows=0) == ns(cols=0) == ns(rows=(1 << 16) + 1) == ns(rows=1 << 16, cols=1 << 15, g=t(ld=1 << 15), out=t(ld=1 << 15)) == BAD
    assert ns(steps=0) == ns(steps=65) == ns(a=float("nan")) == ns(b=float("inf")) == ns(eps=-1.0) == ns(eps=float("nan")) == ns(scale=float("inf")) == BAD
    assert ns(g=None) == ns(out=None) == ns(g=t(data=None)) == ns(out=t(data=None)) == ns(g=t(ld=95)) == ns(out=t(ld=96, f32=3)) == ns(g=t(ld=96, data=FAKE + 1)) == ns(g=t(ld=1 << 26)) == ns(out=t(ld=1 << 26)) == BAD
    assert ns(ws=None) == ns(ws=FAKE + 128) == ns(size=1000) == SPACE
    assert ah.lib().adahop_newton_schulz_workspace_bytes(0, 5) == 0
    assert muon(rows=63) == muon(cols=95) == muon(method_rows=0) == BAD
    w32, w16 = t(ld=96, f32=1), t(ld=96)
    assert muon(momentum=w16) == muon(momentum_out=w16) == muon(w=w16) == muon(w_out=w16) == muon(w_bf16=w32) == BAD
    for name in ("g", "momentum", "momentum_out", "w", "w_out"):
        assert muon(**{name: t(data=None, ld=96, f32=1)}) == BAD
    assert muon(rate=float("nan")) == muon(mu=float("inf")) == muon(weight_decay=float("nan")) == muon(nesterov=2) == BAD
    assert muon(ws=None) == muon(size=1000) == SPACE


def test_binding_refuses_shapes_and_types():
    h, w, y, r = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(9, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    for call in (lambda: ah.adahop_linear_ce(h, w[:, :32], y), lambda: ah.adahop_linear_ce(h, w, y[:3]), lambda: ah.adahop_linear_ce(h, w, y, loss=torch.zeros(3)),
                 lambda: ah.adahop_linear_ce(h, w.t().contiguous().t(), y), lambda: ah.adahop_linear_ce_backward(h, w, y, r[:2]),
                 lambda: ah.adahop_linear_ce_backward(h, w, y, r, torch.zeros(5)), lambda: ah.adahop_linear_ce_backward(h, w, y, r, torch.zeros(8)[::2]),
                 lambda: ah.adahop_linear_ce_backward(h, w, y, r, d_w=w[:4]), lambda: ah.adahop_linear_ce_backward(h, w, y, r, d_h=h, want_h=False),
                 lambda: ah.adahop_linear_ce_backward(h, w, y, r, add=w, want_w=False), lambda: ah.adahop_orthogonalize(h, out=h[:2]), lambda: ah.adahop_orthogonalize(r),
                 lambda: ah.adahop_muon_update(w, h, w, 0.1), lambda: ah.adahop_orthogonalize(h, steps=1 << 40)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ah.adahop_linear_ce(h.float(), w, y), lambda: ah.adahop_linear_ce(h, w, y.int()), lambda: ah.adahop_linear_ce_backward(h, w, y, None),
                 lambda: ah.adahop_orthogonalize(h, dtype=torch.float16), lambda: ah.adahop_orthogonalize(h.half()), lambda: ah.adahop_muon_update(w, w, None, 0.1)):
        with pytest.raises((TypeError, ah.AdahopError)):
            call()


def test_binding_refuses_tensors_in_host_memory():
    h, y, r = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    m = torch.zeros(4, 64)
    for call in (lambda: ah.adahop_linear_ce(h, h, y), lambda: ah.adahop_linear_ce_backward(h, h, y, r), lambda: ah.adahop_orthogonalize(h),
                 lambda: ah.adahop_muon_update(m, h, m, 0.1)):
        with pytest.raises(ValueError, match="on a GPU"):
            call()
