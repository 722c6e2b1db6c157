"""The training operators without a GPU: their 64-bit definitions against differences and against what the format says, and
what the entry points refuse before any GPU work."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import training as orc
from paper_2604_02525_amd import binding as ah

BAD, SPACE = ah.ADAHOP_E_INVALID_ARG, ah.ADAHOP_E_WORKSPACE
FAKE = 0x10000  # never read on these paths


def slope(f, v, at, step=1e-5):
    w = v.copy()
    w[at] += step
    up = f(w)
    w[at] -= 2 * step
    return (up - f(w)) / (2 * step)


@pytest.mark.parametrize("post_norm,gate_rows", [(True, None), (True, 0), (True, 1), (True, 2), (False, 2), (False, None)])
def test_block_norm_gradients_are_the_slopes(post_norm, gate_rows):
    """A central difference of step 1e-5 is 1e-10 times a third derivative off, and rounds at 1e-16 / 1e-5."""
    rng = np.random.default_rng(5)
    rows, cols = 5, 12
    v = dict(x=rng.normal(size=(rows, cols)), y=rng.normal(size=(rows, cols)), w_post=rng.normal(size=cols), w_pre=rng.normal(size=cols),
             gate=None if gate_rows is None else rng.normal(size=cols) if gate_rows == 0 else rng.normal(size=(-(-rows // gate_rows), cols)))
    more = dict(gate_rows=gate_rows or 1, alpha=0.7, beta=1.3, post_norm=post_norm)
    d_s, d_h = rng.normal(size=(rows, cols)), rng.normal(size=(rows, cols))

    def value(**changed):
        r = orc.block_norm(**{**v, **changed}, eps=1e-3, **more)
        return (r["s"] * d_s).sum() + (r["h"] * d_h).sum()

    r = orc.block_norm(**v, eps=1e-3, **more)
    # the means' epsilon enters the formulas through the saved factors alone
    got, _ = orc.block_norm_backward(d_s, d_h, r["shat"], r["yhat"], r["r_s"], r["r_y"], v["w_post"], v["w_pre"], v["gate"], **more)
    for name in ("x", "y", "w_post", "w_pre") + (("gate",) if gate_rows is not None else ()):
        for at in list(np.ndindex(v[name].shape))[::3]:
            assert abs(got["d_" + name][at] - slope(lambda w: value(**{name: w}), v[name], at)) < 1e-7, (name, at)


def test_swiglu_gradients_are_the_slopes():
    rng = np.random.default_rng(6)
    g, u, d_a = (rng.normal(size=(3, 9)) * 2 for _ in range(3))
    d_g, d_u = orc.swiglu_backward(g, u, d_a)
    for at in np.ndindex(g.shape):
        assert abs(d_g[at] - slope(lambda w: (orc.swiglu(w, u) * d_a).sum(), g, at)) < 1e-7
        assert abs(d_u[at] - slope(lambda w: (orc.swiglu(g, w) * d_a).sum(), u, at)) < 1e-7


def test_e4m3_codes_are_those_of_torch():
    """Values and roundings of the element type against an implementation apart from this one."""
    codes = np.arange(256, dtype=np.uint8)
    there = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(orc.E4M3, there, equal_nan=True)
    rng = np.random.default_rng(7)
    mids = (orc.E4M3[:126] + orc.E4M3[1:127]) / 2
    q = np.concatenate([rng.normal(size=4000) * np.exp2(rng.uniform(-12, 9, 4000)), mids, mids * (1 + 2.0 ** -20), mids * (1 - 2.0 ** -20)])
    q = np.clip(np.concatenate([q, -q]), -448, 448).astype(np.float32)
    assert np.array_equal(orc.e4m3_encode(q.astype(np.float64)), torch.from_numpy(q).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_checkpoint_scales():
    x = np.zeros((8, 40))
    x[1, 3], x[2, 3], x[3, 35], x[4, 0], x[5, 0], x[6, :2] = 256.0, 511.9, -1.0, 2.0 ** -130, 3e38, (np.inf, 1.0)
    codes, scales = orc.ckpt8_pack(x)
    assert scales[:, 0].tolist() == [0, 127, 127, 0, 0, 246, 119, 0]
    assert scales[3, 1] == 119 and codes[3, 35] == 0x80 | 0x78          # -256
    assert orc.ckpt8_unpack(codes, scales)[2, 3] == 448.0
    assert codes[6, 0] == 127 and orc.ckpt8_unpack(codes, scales)[6, 1] == 1.0


# ---- refusals ---------------------------------------------------------------------------------------------------------------
def t(ld=64, f32=0, data=FAKE):
    return ah.adahop_tensor_t(data, ld, f32)


def k(ld=64, ls=2, codes=FAKE, scales=FAKE):
    return ah.adahop_ckpt8_t(codes, scales, ld, ls)


def test_checkpoints_refuse():
    L = ah.lib()
    pack = lambda rows=4, cols=64, x=t(), out=k(): L.adahop_ckpt8_pack(rows, cols, x and C.byref(x), out and C.byref(out), None)  # noqa: E731
    unpack = lambda rows=4, cols=64, x=k(), w=None, out=t(): L.adahop_ckpt8_unpack(rows, cols, C.byref(x), w and C.byref(w), C.byref(out), None)  # noqa: E731
    for f in (pack, unpack):
        assert f(rows=-1) == f(cols=0) == f(rows=(1 << 21) + 1) == f(cols=(1 << 21) + 1) == f(rows=1 << 20, cols=1 << 16) == BAD
        assert f(rows=0) == ah.ADAHOP_OK
    assert pack(x=None) == pack(out=None) == pack(x=t(data=None)) == pack(x=t(ld=63)) == pack(x=t(f32=2)) == pack(x=t(data=FAKE + 1)) == BAD
    assert pack(x=t(f32=1, data=FAKE + 2)) == BAD
    for bad in (k(ld=63), k(ld=72), k(ls=1), k(codes=FAKE + 8), k(codes=None), k(scales=None)):
        assert pack(out=bad) == unpack(x=bad) == BAD
    assert unpack(w=t(data=FAKE + 1)) == unpack(out=t(ld=32)) == unpack(out=t(data=None)) == BAD


def swiglu(**more):
    p = ah.adahop_swiglu_t(4, 64, t(), t(), t())
    p.d_a, p.d_g, p.d_u = t(), t(), t()
    for name, v in more.items():
        setattr(p, name, v)
    return p


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(cols=0), dict(g=t(ld=32)), dict(u=t(data=FAKE + 1)), dict(g=t(data=None)), dict(a=t(ld=8)),
                                 dict(ckpt_g=k(ld=32), ckpt_u=k())])
def test_swiglu_refuses(bad):
    L = ah.lib()
    assert L.adahop_swiglu(C.byref(swiglu(**bad)), None) == BAD
    assert L.adahop_swiglu_backward(C.byref(swiglu(**bad)), None) == BAD


def test_swiglu_refuses_in_one_direction():
    L = ah.lib()
    assert L.adahop_swiglu(None, None) == L.adahop_swiglu_backward(None, None) == BAD
    assert L.adahop_swiglu(C.byref(swiglu(g=t(f32=1))), None) == BAD                        # g and u of two types
    assert L.adahop_swiglu(C.byref(swiglu(a=t(data=None))), None) == BAD
    for bad in (dict(ckpt_g=k()), dict(ckpt_u=k()), dict(d_a=t(data=None)), dict(d_g=t(data=None)), dict(d_u=t(ld=63)), dict(ckpt_a=k(ls=1))):
        assert L.adahop_swiglu_backward(C.byref(swiglu(**bad)), None) == BAD
    for f in (L.adahop_swiglu, L.adahop_swiglu_backward):
        assert f(C.byref(swiglu(rows=0, g=t(data=None), u=t(data=None))), None) == ah.ADAHOP_OK


def norm(**more):
    p = ah.adahop_block_norm_t(4, 64, 1, 1e-6, 1.0, 1.0, t(), t(), t(), t())
    p.s, p.h, p.rstd_post, p.rstd_pre = t(), t(), FAKE, FAKE
    p.d_s, p.d_h, p.d_x, p.d_y = t(), t(), t(), t()
    for name, v in more.items():
        setattr(p, name, v)
    return p


BOTH_WAYS = [dict(rows=-1), dict(cols=0), dict(cols=16385), dict(post_norm=2), dict(residual_scale=float("inf")), dict(branch_scale=float("nan")),
             dict(w_post=t(data=FAKE + 1)), dict(w_pre=t(f32=3)), dict(gate=t(), gates=1, gate_rows=3), dict(gate=t(), gates=4, gate_rows=0),
             dict(gate=t(ld=32), gates=1, gate_rows=4), dict(gate=t(), gates=-1, gate_rows=4), dict(rstd_post=FAKE + 2), dict(rstd_pre=FAKE + 1),
             dict(x=t(ld=8)), dict(y=t(f32=7)), dict(s=t(data=FAKE + 1)), dict(h=t(ld=63)), dict(ckpt_y=k(ld=8), ckpt_s=k()),
             dict(ckpt_y=k(), ckpt_s=k(scales=None))]


@pytest.mark.parametrize("bad", BOTH_WAYS)
def test_block_norm_refuses(bad):
    L = ah.lib()
    assert L.adahop_block_norm(C.byref(norm(**bad)), None) == BAD
    assert L.adahop_block_norm_backward(C.byref(norm(**bad)), FAKE, 1 << 30, None) == BAD


def test_block_norm_refuses_in_one_direction():
    L = ah.lib()
    none = t(data=None)
    assert L.adahop_block_norm(None, None) == L.adahop_block_norm_backward(None, None, 0, None) == BAD
    for bad in (dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=none, y=none, post_norm=0), dict(s=none, h=none),
                dict(s=t(f32=1)), dict(y=none), dict(y=none, post_norm=0, gate=t(), gates=1, gate_rows=4), dict(y=none, post_norm=0, ckpt_y=k()),
                dict(post_norm=0), dict(h=none), dict(h=none, rstd_pre=None, ckpt_s=k())):
        assert L.adahop_block_norm(C.byref(norm(**bad)), None) == BAD, bad
    back = lambda **bad: L.adahop_block_norm_backward(C.byref(norm(**bad)), FAKE, 1 << 30, None)  # noqa: E731
    for bad in (dict(d_gate=t()), dict(d_s=none, d_h=none), dict(rstd_pre=None), dict(s=none), dict(d_h=none, d_w_pre=FAKE), dict(y=none),
                dict(rstd_post=None), dict(ckpt_s=k()), dict(ckpt_y=k()), dict(d_x=t(f32=1)), dict(d_s=t(f32=1)), dict(s=t(f32=1)), dict(d_y=t(f32=1)),
                dict(d_h=t(f32=1)), dict(y=t(f32=1)), dict(d_x=t(ld=3)), dict(d_w_post=FAKE + 1)):
        assert back(**bad) == BAD, bad
    need = L.adahop_block_norm_backward_workspace_bytes(4, 64, 0)
    assert need > 0 and need % 4 == 0
    for ws, size in ((None, need), (FAKE + 16, need), (FAKE, need - 1)):
        assert L.adahop_block_norm_backward(C.byref(norm()), ws, size, None) == SPACE
    assert L.adahop_block_norm_backward_workspace_bytes(0, 64, 0) == L.adahop_block_norm_backward_workspace_bytes(4, 16385, 0) == 0
    assert L.adahop_block_norm(C.byref(norm(rows=0)), None) == ah.ADAHOP_OK


def wgrad(T=8, N=64, D=64, G=t(), x=k(), w=None, add=None, C_=t(f32=1), ws=FAKE, size=1 << 40):
    r = lambda v: v and C.byref(v)  # noqa: E731
    return ah.lib().adahop_ckpt8_wgrad(T, N, D, r(G), r(x), r(w), r(add), r(C_), ws, size, None)


def test_wgrad_refuses():
    assert wgrad(T=-1) == wgrad(N=0) == wgrad(D=0) == wgrad(T=(1 << 21) + 1) == wgrad(N=1 << 20, D=1 << 16) == BAD
    assert wgrad(G=None) == wgrad(x=None) == wgrad(C_=None) == BAD
    assert wgrad(G=t(f32=1)) == wgrad(G=t(ld=68)) == wgrad(G=t(ld=56)) == wgrad(G=t(data=FAKE + 8)) == wgrad(G=t(data=None)) == BAD
    assert wgrad(G=t(ld=1 << 25)) == wgrad(x=k(ld=1 << 25)) == wgrad(x=k(ls=1 << 25)) == BAD
    assert wgrad(x=k(ld=48)) == wgrad(x=k(ls=1)) == wgrad(x=k(codes=FAKE + 4)) == wgrad(x=k(codes=None)) == wgrad(x=k(codes=None, scales=None)) == BAD
    assert wgrad(C_=t(data=None)) == wgrad(C_=t(ld=63)) == wgrad(w=t(data=FAKE + 1)) == wgrad(add=t(ld=8)) == wgrad(add=t(f32=5)) == BAD
    L = ah.lib()
    need = L.adahop_ckpt8_wgrad_workspace_bytes(32768, 64, 64)
    if need:
        assert wgrad(T=32768, ws=None, size=need) == wgrad(T=32768, ws=FAKE + 16, size=need) == wgrad(T=32768, size=need - 1) == SPACE
    assert L.adahop_ckpt8_wgrad_workspace_bytes(8, 0, 64) == 0


def test_binding_refuses_shapes_and_types():
    x, y = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 64, dtype=torch.bfloat16)
    codes, scales = ah.adahop_ckpt8_empty(4, 64, "cpu")
    with pytest.raises(ValueError):
        ah.adahop_block_norm(x, y[:3])
    with pytest.raises(ValueError):
        ah.adahop_block_norm(x, y, w_post=torch.zeros(63))
    with pytest.raises(TypeError):
        ah.adahop_block_norm(x, y, w_pre=torch.zeros(64, dtype=torch.float16))
    with pytest.raises(ValueError):
        ah.adahop_block_norm(x, y, keep="everything")
    with pytest.raises(ValueError):
        ah.adahop_block_norm(x, y.t().contiguous().t())
    with pytest.raises(ValueError):
        ah.adahop_swiglu(x, y[:, :32])
    with pytest.raises(ValueError):
        ah.adahop_swiglu_backward((codes[:, :32], scales), (codes, scales), x)
    with pytest.raises(ValueError):
        ah.adahop_ckpt8_wgrad(x[:3], (codes, scales))
    with pytest.raises(ValueError):
        ah.adahop_ckpt8_unpack((codes, scales[:, :1]))
    with pytest.raises(TypeError):
        ah.adahop_ckpt8_pack(x.to(torch.float64))
    with pytest.raises(ValueError):
        ah.adahop_block_norm_backward(x, y, x, y, torch.zeros(3), torch.zeros(4))


def test_binding_refuses_tensors_in_host_memory():
    x, r = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4)
    pair = ah.adahop_ckpt8_empty(4, 64, "cpu")
    for call in (lambda: ah.adahop_ckpt8_pack(x), lambda: ah.adahop_ckpt8_unpack(pair), lambda: ah.adahop_swiglu(x, x),
                 lambda: ah.adahop_swiglu_backward(x, x, x), lambda: ah.adahop_block_norm(x, x),
                 lambda: ah.adahop_block_norm_backward(x, x, x, x, r, r), lambda: ah.adahop_ckpt8_wgrad(x, pair)):
        with pytest.raises(ValueError, match="on a GPU"):
            call()


def test_binding_refuses_what_is_no_stream():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    for stream in ("0", 1.5, object()):
        with pytest.raises(TypeError, match="stream"):
            ah.adahop_ckpt8_pack(x, stream=stream)
