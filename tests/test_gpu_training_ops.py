"""The training operators on the GPU against their 64-bit definitions (oracle/training.py).

Bounds.  A bf16 output is rounded once: half a step, at most 2^-8 of its value.  Before that everything is in fp32: an output
that is a sum of terms of total magnitude m, formed in a handful of operations from a row's sums (of at most 16384 terms in some 2^10 threads: a chain of
16 additions in a thread and 10 between them), is off by less than EPS * m with EPS = 64 * 2^-24.  Sums over rows are chains of at most
`rows` additions.  What is held in 8 bits and comes from bf16 or fp32 inputs without arithmetic is compared bit for bit; the codes of a normalised value may fall to
the other side of a tie or of a power of two, so there the value may be half a step (1/16 of it, or half of 2^-9 times the scale) and EPS
off, and what saturates (448 to 512 times the scale) an eighth of it."""
import numpy as np
import pytest

from oracle import training as orc

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

EPS = 64 * 2.0 ** -24
BF16 = 2.0 ** -8


@pytest.fixture(scope="module")
def ah():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_02525_amd import binding
    binding.lib()
    return binding


def say(*a):
    print("[case]", *a, flush=True)


def up(a, f32=False, pad=0, offset=0):
    """A numpy array as a GPU tensor, rows `pad` elements further apart than they are long and beginning `offset` elements into memory."""
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a)).to(torch.float32 if f32 else torch.bfloat16)
    if not pad and not offset:
        return t.cuda()
    if t.dim() == 1:
        t = t[None]
    room = torch.full((t.shape[0] * (t.shape[1] + pad) + offset,), float("nan"), dtype=t.dtype, device="cuda")
    v = room[offset:].view(t.shape[0], t.shape[1] + pad)[:, :t.shape[1]]
    v.copy_(t)
    return v


def room_for(rows, cols, dtype, pad):
    """Where an output goes: rows `pad` apart, and all of it, to see what lies around it untouched."""
    all_of_it = torch.full((rows, cols + pad), 7, dtype=dtype, device="cuda")
    return all_of_it[:, :cols], all_of_it[:, cols:]


def down(t):
    return t.detach().double().cpu().numpy()


def bf16(a):
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16).double().numpy()


def close(got, want, mag, f32, what, chain=1):
    """|got - want| within EPS * chain * mag and, in bf16, half a step."""
    off = np.abs(down(got) - want)
    bound = EPS * chain * mag + (0.0 if f32 else BF16 * np.abs(want)) + 1e-37
    worst = np.unravel_index(np.argmax(off - bound), off.shape)
    assert np.all(off <= bound), f"{what}: {off[worst]:.3e} off where {bound[worst]:.3e} is allowed, at {worst}"


def stored8(pair):
    return pair[0].cpu().numpy(), pair[1].cpu().numpy()


def close8(pair, want, mag, what):
    codes, scales = stored8(pair)
    each = np.repeat(np.exp2(scales.astype(np.float64) - 127), 32, axis=1)[:, :codes.shape[1]]
    got = orc.ckpt8_unpack(codes, scales)
    bound = np.abs(want) / 16 + each * 2.0 ** -10 + EPS * mag
    bound = np.where(np.abs(want) > 448 * each, np.abs(want) / 8 + EPS * mag, bound)
    assert np.all(np.abs(got - want) <= bound * (1 + 1e-9)), what
    amax = np.abs(want).max(1)
    assert np.all(amax <= 512.01 * each.max(1)) and np.all((amax >= 255.9 * each.max(1)) | (each.max(1) <= 2.0 ** -126)), what


# ---- 8-bit checkpoints ---------------------------------------------------------------------------------------------------------
def special_rows():
    """Rows of 64 that hold what the format treats apart."""
    rng = np.random.default_rng(1)
    rows = [np.zeros(64), -np.zeros(64), rng.normal(size=64), rng.normal(size=64) * 1e-30, rng.normal(size=64) * 1e30]
    ties = (orc.E4M3[:126] + orc.E4M3[1:127]) / 2                       # between neighbouring codes, in blocks whose scale is 1 (256 comes first)
    for part in np.split(np.concatenate([ties, ties[:60]])[:186], 6):
        rows += [np.concatenate([[256.0], part, [300.0], part]), -np.concatenate([[256.0], part, [300.0], part])]
    rows += [np.full(64, 2.0 ** -133), np.full(64, 3e38), np.concatenate([[1.0, np.inf], np.ones(30), [np.nan, 2.0], np.ones(30)]),
             np.full(64, np.inf), np.full(64, -np.nan), np.concatenate([[3e38, -np.inf], np.zeros(62)]), np.full(64, 449.0), np.full(64, 511.0)]
    return np.stack([r[:64] for r in rows])


@pytest.mark.parametrize("f32", [False, True])
def test_pack_of_special_values(ah, f32):
    x = special_rows()
    t = up(x, f32)
    x = down(t)
    say("pack", x.shape, f32)
    codes, scales = stored8(ah.adahop_ckpt8_pack(t))
    want_c, want_s = orc.ckpt8_pack(x)
    nan = want_c & 127 == 127
    assert np.array_equal(scales, want_s)
    assert np.array_equal(codes[~nan], want_c[~nan]) and np.all(codes[nan] & 127 == 127)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (2, 33), (3, 64), (7, 100), (5, 515), (257, 96), (33, 4091), (64, 8192), (1, 28672)])
@pytest.mark.parametrize("f32,pad,offset", [(False, 0, 0), (True, 0, 0), (False, 5, 1), (True, 3, 1)])
def test_pack_and_unpack(ah, rows, cols, f32, pad, offset):
    rng = np.random.default_rng(rows * 31 + cols)
    x = rng.normal(size=(rows, cols)) * np.exp2(rng.integers(-6, 7, size=(rows, cols)))
    t = up(x, f32, pad, offset)
    x = down(t)
    say("pack / unpack", rows, cols, f32, pad, offset)
    pair = ah.adahop_ckpt8_empty(rows, cols)
    whole = torch.full((rows, pair[0].stride(0) if rows > 1 else (cols + 15) // 16 * 16), 0x55, dtype=torch.uint8, device="cuda")
    pair = (whole[:, :cols], pair[1])
    ah.adahop_ckpt8_pack(t, out=pair)
    codes, scales = stored8(pair)
    want_c, want_s = orc.ckpt8_pack(x)
    assert np.array_equal(codes, want_c) and np.array_equal(scales, want_s)
    assert torch.all(whole[:, cols:] == 0x55), "bytes past the columns were written"
    value = orc.ckpt8_unpack(want_c, want_s)
    w = bf16(1 + 0.2 * rng.normal(size=cols))
    for o32 in (False, True):
        out, around = room_for(rows, cols, torch.float32 if o32 else torch.bfloat16, pad)
        ah.adahop_ckpt8_unpack(pair, out=out)
        assert np.array_equal(down(out), value) and torch.all(around == 7)
        ah.adahop_ckpt8_unpack(pair, col_scale=up(w, o32), out=out)
        close(out, value * w, np.abs(value * w), o32, "unpack with a weight")


def test_unpack_of_every_code_and_scale(ah):
    codes = np.tile(np.repeat(np.arange(256, dtype=np.uint8).reshape(8, 32), 1, axis=0).reshape(1, 256), (255, 1))
    scales = np.tile(np.arange(255, dtype=np.uint8)[:, None], (1, 8))
    say("unpack, all codes and scales")
    out = down(ah.adahop_ckpt8_unpack((torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()), dtype=torch.float32))
    with np.errstate(over="ignore"):
        want = orc.ckpt8_unpack(codes, scales).astype(np.float32).astype(np.float64)    # beyond 2^128: infinite
    assert np.array_equal(out, want, equal_nan=True)


# ---- gated activation ------------------------------------------------------------------------------------------------------------
def act_error(g):
    """Of silu and its slope in fp32, as a multiple of 2^-24: exp's argument is rounded at |g| log2(e), a few operations follow."""
    return (2 * np.abs(g) + 16) * 2.0 ** -24


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 33), (2, 515), (40, 100), (9, 4091), (16, 14336)])
@pytest.mark.parametrize("f32,pad", [(False, 0), (True, 0), (False, 3), (True, 1)])
def test_swiglu(ah, rows, cols, f32, pad):
    rng = np.random.default_rng(rows + cols)
    both = up(np.concatenate([rng.normal(size=(rows, cols)) * 3, rng.normal(size=(rows, cols))], 1), f32, pad)
    g, u = both[:, :cols], both[:, cols:]
    g64, u64 = down(g), down(u)
    if cols > 8:
        g[0, 3], g[0, 5] = 120.0, -120.0
        g64 = down(g)
    for a32 in (False, True):
        a, around = room_for(rows, cols, torch.float32 if a32 else torch.bfloat16, pad)
        say("swiglu", rows, cols, f32, pad, a32)
        r = ah.adahop_swiglu(g, u, a=a, keep8=True)
        want = orc.swiglu(g64, u64)
        off = np.abs(down(a) - want)
        assert np.all(off <= (act_error(g64) + (0 if a32 else BF16)) * np.abs(want) + 1e-37) and torch.all(around == 7)
        for name, v in (("ckpt_g", g64), ("ckpt_u", u64)):
            c, s = orc.ckpt8_pack(v)
            assert np.array_equal(stored8(r[name])[0], c) and np.array_equal(stored8(r[name])[1], s), name
    assert torch.equal(ah.adahop_swiglu(g, u)["a"], ah.adahop_swiglu(g, u, a=torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda"))["a"])


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 33), (2, 515), (40, 100), (9, 4091), (16, 14336)])
@pytest.mark.parametrize("kept,f32,pad", [(True, False, 0), (True, True, 3), (False, False, 1), (False, True, 0)])
def test_swiglu_backward(ah, rows, cols, kept, f32, pad):
    rng = np.random.default_rng(rows * 7 + cols)
    g, u = up(rng.normal(size=(rows, cols)) * 3, pad=pad), up(rng.normal(size=(rows, cols)), pad=pad)
    d_a = up(rng.normal(size=(rows, cols)) * 1e-3, f32, pad)
    g64, u64, da64 = down(g), down(u), down(d_a)
    if kept:
        g, u = ah.adahop_ckpt8_pack(g), ah.adahop_ckpt8_pack(u)
        g64, u64 = orc.ckpt8_unpack(*stored8(g)), orc.ckpt8_unpack(*stored8(u))
    want_g, want_u = orc.swiglu_backward(g64, u64, da64)
    want_a = orc.swiglu(g64, u64)
    say("swiglu backward", rows, cols, kept, f32, pad)
    slope = np.abs(da64 * u64) * (1 / (1 + np.exp(-g64)) + np.abs(g64) / (1 + np.exp(-g64)))
    a8 = ah.adahop_ckpt8_empty(rows, cols)
    r = ah.adahop_swiglu_backward(g, u, d_a, a=a8)
    assert np.all(np.abs(down(r["d_g"]) - want_g) <= act_error(g64) * slope + BF16 * np.abs(want_g) + 1e-37)
    assert np.all(np.abs(down(r["d_u"]) - want_u) <= (act_error(g64) + BF16) * np.abs(want_u) + 1e-37)
    if rows > 1:
        assert r["d_u"].data_ptr() == r["d_g"].data_ptr() + 2 * cols and r["d_g"].stride(0) == 2 * cols
    close8(a8, want_a, np.abs(want_a) * (1 + act_error(g64) / EPS), "a in 8 bits")
    out = {n: torch.empty(rows, cols, dtype=torch.float32, device="cuda") for n in ("d_g", "d_u", "a")}
    r = ah.adahop_swiglu_backward(g, u, d_a, **out)
    assert np.all(np.abs(down(r["d_g"]) - want_g) <= act_error(g64) * slope + 1e-37)
    assert np.all(np.abs(down(r["d_u"]) - want_u) <= act_error(g64) * np.abs(want_u) + 1e-37)
    assert np.all(np.abs(down(r["a"]) - want_a) <= act_error(g64) * np.abs(want_a) + 1e-37)
    if not kept:            # the gradients in the place of what they are of
        alone = ah.adahop_swiglu_backward(g, u, d_a)
        d_g, d_u = down(alone["d_g"]), down(alone["d_u"])
        ah.adahop_swiglu_backward(g, u, d_a, d_g=g, d_u=u)
        assert np.array_equal(down(g), d_g) and np.array_equal(down(u), d_u)


# ---- block norm --------------------------------------------------------------------------------------------------------------------
SHAPES = [(1, 1), (1, 7), (3, 64), (5, 100), (2, 512), (9, 520), (7, 4091), (64, 2048), (33, 8192), (5, 8200), (3, 16384), (300, 96), (2100, 64)]
GATES = [None, "vector", 3, 1, 700]


def norm_inputs(rows, cols, gate, seed):
    rng = np.random.default_rng(seed)
    x, y = rng.normal(size=(rows, cols)), rng.normal(size=(rows, cols)) * 2
    y[:, rng.integers(0, cols, 2)] *= 30
    if rows > 2:
        y[1] = 0            # a row of zeros
        x[2] = 0
    v = dict(x=bf16(x), y=bf16(y), w_post=bf16(1 + 0.2 * rng.normal(size=cols)), w_pre=bf16(1 + 0.2 * rng.normal(size=cols)), gate=None)
    rows_per = 1
    if gate == "vector":
        v["gate"] = bf16(rng.normal(size=cols))
    elif gate:
        rows_per, v["gate"] = gate, bf16(rng.normal(size=(-(-rows // gate), cols)))
    return v, rows_per, rng


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("s32,y32,pad", [(False, False, 0), (True, False, 0), (False, True, 3)])
def test_block_norm(ah, rows, cols, gate, s32, y32, pad):
    v, rows_per, _ = norm_inputs(rows, cols, gate, rows + cols)
    alpha, beta, eps = 0.75, 1.5, 1e-5
    want = orc.block_norm(**v, gate_rows=rows_per, alpha=alpha, beta=beta, eps=eps)
    t = {n: up(v[n], f32, pad) for n, f32 in (("x", s32), ("y", y32))}
    s, s_around = room_for(rows, cols, torch.float32 if s32 else torch.bfloat16, pad)
    h, h_around = room_for(rows, cols, torch.float32 if y32 else torch.bfloat16, pad)
    say("block norm", rows, cols, gate, s32, y32, pad)
    r = ah.adahop_block_norm(**t, w_post=up(v["w_post"], s32), w_pre=up(v["w_pre"], y32), gate=up(v["gate"], y32), gate_rows=rows_per,
                             residual_scale=alpha, branch_scale=beta, eps=eps, s=s, h=h, keep="ckpt8")
    branch = beta * orc.gate_of_rows(v["gate"], rows_per, rows) * v["w_post"] * want["yhat"]
    mag = np.abs(alpha * v["x"]) + np.abs(branch)
    # the root mean square of s inherits the errors of its elements
    rel = 1 + np.sqrt((mag ** 2).mean(1) / ((want["s"] ** 2).mean(1) + eps))
    close(r["s"], want["s"], mag, s32, "s")
    shat_mag = want["r_s"][:, None] * mag + np.abs(want["shat"]) * rel[:, None]
    close(r["h"], want["h"], np.abs(v["w_pre"]) * shat_mag, y32, "h")
    close(r["rstd_post"], want["r_y"], want["r_y"], True, "rstd_post")
    close(r["rstd_pre"], want["r_s"], want["r_s"] * rel, True, "rstd_pre")
    close8(r["ckpt_y"], want["yhat"], np.abs(want["yhat"]), "ckpt_y")
    close8(r["ckpt_s"], want["shat"], shat_mag, "ckpt_s")
    assert torch.all(s_around == 7) and torch.all(h_around == 7)


@pytest.mark.parametrize("rows,cols", [(1, 64), (3, 1000), (5, 8200)])
def test_block_norm_forms(ah, rows, cols):
    """Without a residual, without a post norm, without weights, before the first block, after the last, and in place."""
    v, _, rng = norm_inputs(rows, cols, None, rows * 3 + cols)
    x, y, w = up(v["x"]), up(v["y"]), up(v["w_pre"])
    say("block norm forms", rows, cols)
    first = orc.block_norm(v["x"], None, None, v["w_pre"])
    r = ah.adahop_block_norm(x, w_pre=w, keep="ckpt8")
    assert r["s"] is x and r["ckpt_y"] is None and r["rstd_post"] is None
    close(r["h"], first["h"], 4 * np.abs(first["h"]), False, "h of x")
    close8(r["ckpt_s"], first["shat"], 4 * np.abs(first["shat"]), "ckpt_s of x")
    r = ah.adahop_block_norm(x, residual_scale=2.0)
    close(r["s"], 2 * v["x"], np.abs(v["x"]), False, "scaled x") if r["s"] is not x else None
    last = orc.block_norm(v["x"], v["y"], None, None)
    r = ah.adahop_block_norm(x, y, pre_norm=False)
    assert r["h"] is None
    close(r["s"], last["s"], np.abs(v["x"]) + np.abs(last["yhat"]), False, "s without h")
    plain = orc.block_norm(v["x"], v["y"], v["w_post"], v["w_pre"], post_norm=False)
    mag = np.abs(v["x"]) + np.abs(v["y"] * v["w_post"])
    r = ah.adahop_block_norm(x, y, w_post=up(v["w_post"]), w_pre=w, post_norm=False, keep="ckpt8")
    assert r["rstd_post"] is None
    close(r["s"], plain["s"], mag, False, "s without a post norm")
    c, sc = orc.ckpt8_pack(v["y"])
    assert np.array_equal(stored8(r["ckpt_y"])[0], c) and np.array_equal(stored8(r["ckpt_y"])[1], sc)
    alone = orc.block_norm(None, v["y"], v["w_post"], v["w_pre"])
    r = ah.adahop_block_norm(None, y, w_post=up(v["w_post"]), w_pre=w)
    close(r["s"], alone["s"], np.abs(alone["s"]), False, "s without a residual")
    want = ah.adahop_block_norm(x, y, w_pre=w)
    r = ah.adahop_block_norm(x, y, w_pre=w, s=x)
    assert r["s"] is x and torch.equal(x, want["s"]) and torch.equal(r["h"], want["h"])


def saved_for_backward(ah, v, rows_per, rng, kept, s32, y32, pad, alpha, beta, post_norm=True):
    """What the forward pass leaves, as tensors and in 64 bits: (s, y, rstd_pre, rstd_post), dict(shat, yhat, r_s, r_y)."""
    f = orc.block_norm(**v, gate_rows=rows_per, alpha=alpha, beta=beta, eps=1e-5, post_norm=post_norm)
    r_s, r_y = up(f["r_s"], True), up(f["r_y"], True)
    d = dict(r_s=down(r_s), r_y=down(r_y))
    if kept:
        s, y = ah.adahop_ckpt8_pack(up(f["shat"], True)), ah.adahop_ckpt8_pack(up(f["yhat"], True))
        d.update(shat=orc.ckpt8_unpack(*stored8(s)), yhat=orc.ckpt8_unpack(*stored8(y)))
    else:
        s, y = up(f["s"], s32, pad), up(v["y"], y32, pad)
        d.update(shat=down(s) * d["r_s"][:, None], yhat=down(y) * d["r_y"][:, None])
    return (s, y, r_s, r_y if post_norm else None), d


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("kept,s32,y32,pad", [(True, False, False, 0), (False, False, False, 0), (True, True, True, 3), (False, True, False, 0), (False, False, True, 1)])
def test_block_norm_backward(ah, rows, cols, gate, kept, s32, y32, pad):
    v, rows_per, rng = norm_inputs(rows, cols, gate, rows * 5 + cols)
    alpha, beta = 0.75, 1.5
    saved, d = saved_for_backward(ah, v, rows_per, rng, kept, s32, y32, pad, alpha, beta)
    d_s, d_h = up(rng.normal(size=(rows, cols)) * 1e-3, s32, pad), up(rng.normal(size=(rows, cols)) * 1e-3, y32, pad)
    want, mag = orc.block_norm_backward(down(d_s), down(d_h), **d, w_post=v["w_post"], w_pre=v["w_pre"], gate=v["gate"], gate_rows=rows_per, alpha=alpha,
                                        beta=beta)
    more = dict(w_post=up(v["w_post"]), w_pre=up(v["w_pre"]), gate=up(v["gate"], y32), gate_rows=rows_per, residual_scale=alpha, branch_scale=beta)
    d_x, x_around = room_for(rows, cols, d_s.dtype, pad)
    d_y, y_around = room_for(rows, cols, d_h.dtype, pad)
    say("block norm backward", rows, cols, gate, kept, s32, y32, pad)
    r = ah.adahop_block_norm_backward(d_s, d_h, *saved, **more, d_x=d_x, d_y=d_y)
    for name, m in mag.items():
        f32 = {"d_x": s32, "d_y": y32, "d_gate": y32}.get(name, True)
        # sums over rows: a chain of at most `rows` additions, and of the parts that are added up
        close(r[name], want[name], m, f32, name, chain=1 + (rows / 64 if name in ("d_w_post", "d_w_pre", "d_gate") else 0))
    assert torch.all(x_around == 7) and torch.all(y_around == 7)
    again = ah.adahop_block_norm_backward(d_s, d_h, *saved, **more)
    for name in mag:
        assert torch.equal(again[name], r[name]), f"{name}: other bits in a second call"
    here = ah.adahop_block_norm_backward(d_s, d_h, *saved, **more, d_x=d_s, d_y=d_h)         # in the gradients' own place
    for name in mag:
        assert torch.equal(here[name], r[name]), f"{name}: other bits in place"


@pytest.mark.parametrize("kept", [True, False])
@pytest.mark.parametrize("form", ["no d_s", "no d_h", "no y", "no post norm", "no weights"])
def test_block_norm_backward_forms(ah, kept, form):
    rows, cols = 37, 1000
    v, rows_per, rng = norm_inputs(rows, cols, None, 11)
    if form == "no weights":
        v["w_post"] = v["w_pre"] = None
    post = form != "no post norm"
    saved, d = saved_for_backward(ah, v, 1, rng, kept, False, False, 0, 1.0, 1.0, post)
    d_s, d_h = up(rng.normal(size=(rows, cols)) * 1e-3), up(rng.normal(size=(rows, cols)) * 1e-3)
    if form == "no d_s":
        d_s = None
    if form == "no d_h":
        d_h = None
    s, y, r_s, r_y = saved
    if form == "no y":
        y, d["yhat"] = None, None
    if form == "no d_h":
        s, r_s = None, None
    say("block norm backward,", form, kept)
    r = ah.adahop_block_norm_backward(d_s, d_h, s, y, r_s, r_y, w_post=None if y is None else up(v["w_post"]), w_pre=up(v["w_pre"]), post_norm=post)
    want, mag = orc.block_norm_backward(None if d_s is None else down(d_s), None if d_h is None else down(d_h), **d, w_post=v["w_post"], w_pre=v["w_pre"],
                                        post_norm=post)
    for name, m in mag.items():
        if form == "no weights" and name.startswith("d_w"):
            assert r[name] is None
            continue
        close(r[name], want[name], m, name.startswith("d_w"), name, chain=2)
    if form == "no y":
        assert r["d_y"] is None
    if form == "no d_h":
        assert r["d_w_pre"] is None


def test_infinities_and_nan_stay_in_their_row(ah):
    """A row that holds one makes its own outputs NaN or infinite, and no other's; column sums take them up."""
    rows, cols = 6, 300
    v, _, rng = norm_inputs(rows, cols, None, 12)
    x, y, w = up(v["x"]), up(v["y"]), up(v["w_pre"])
    bad_x, bad_y = x.clone(), y.clone()
    bad_x[3, 7], bad_y[5, 9] = float("inf"), float("nan")
    clean = [i for i in range(rows) if i not in (3, 5)]
    say("block norm with infinities")
    a, b = ah.adahop_block_norm(x, y, w_pre=w, keep="ckpt8"), ah.adahop_block_norm(bad_x, bad_y, w_pre=w, keep="ckpt8")
    for name in ("s", "h", "rstd_post", "rstd_pre"):
        assert torch.equal(a[name][clean], b[name][clean]), name
    assert torch.equal(a["ckpt_s"][0][clean], b["ckpt_s"][0][clean])
    assert bool(b["h"][5].isnan().all()) and bool(torch.all(b["ckpt_s"][0][5] & 127 == 127))
    d = up(rng.normal(size=(rows, cols)))
    bad_d = d.clone()
    bad_d[2, 4] = float("nan")
    back = lambda g: ah.adahop_block_norm_backward(g, g, a["ckpt_s"], a["ckpt_y"], a["rstd_pre"], a["rstd_post"], w_pre=w)  # noqa: E731
    ok, nan = back(d), back(bad_d)
    rest = [i for i in range(rows) if i != 2]
    for name in ("d_x", "d_y"):
        assert torch.equal(ok[name][rest], nan[name][rest]) and bool(nan[name][2].isnan().any())
    assert bool(nan["d_w_pre"][4].isnan()) and int(nan["d_w_pre"].isnan().sum()) == 1


# ---- weight gradient ---------------------------------------------------------------------------------------------------------------
def wgrad_bound(G, x, scale, tokens):
    """fp32 additions of `tokens` exact products in any order, and the two operations behind them."""
    m = np.abs(G).T @ np.abs(x)
    return (2 * tokens + 16) * 2.0 ** -24 * (m if scale is None else m * np.abs(scale))


@pytest.mark.parametrize("tokens", [0, 1, 2, 15, 31, 33, 64, 65, 127, 300])
@pytest.mark.parametrize("d_out,d_in", [(1, 1), (8, 32), (64, 64), (65, 33), (100, 515), (256, 256), (257, 300), (520, 264)])
@pytest.mark.parametrize("scaled,add,bf16_out,pad", [(False, False, False, 0), (True, True, False, 3), (True, False, True, 1), (False, True, True, 0)])
def test_wgrad(ah, tokens, d_out, d_in, scaled, add, bf16_out, pad):
    run_wgrad(ah, tokens, d_out, d_in, scaled, add, bf16_out, pad)


@pytest.mark.parametrize("tokens,d_out,d_in", [(4096, 64, 96), (5001, 40, 40), (1000, 1024, 768), (2048, 264, 1032), (20000, 16, 32)])
def test_wgrad_of_many_tokens(ah, tokens, d_out, d_in):
    run_wgrad(ah, tokens, d_out, d_in, True, True, False, 0)
    run_wgrad(ah, tokens, d_out, d_in, False, False, True, 0)


def run_wgrad(ah, tokens, d_out, d_in, scaled, add, bf16_out, pad):
    rng = np.random.default_rng(tokens * 3 + d_out + d_in)
    ld = (d_out + 7) // 8 * 8 + 8 * (pad > 0)
    G = torch.full((max(tokens, 1), ld), float("nan"), dtype=torch.bfloat16, device="cuda")[:tokens, :d_out]
    G.copy_(torch.from_numpy(rng.normal(size=(tokens, d_out)) * 1e-3))
    x8 = ah.adahop_ckpt8_pack(up(rng.normal(size=(tokens, d_in)) * np.exp2(rng.integers(-4, 5, size=(tokens, 1)))))
    scale = up(1 + 0.2 * rng.normal(size=d_in), not bf16_out) if scaled else None
    more = up(rng.normal(size=(d_out, d_in)) * 1e-2, not bf16_out, pad) if add else None
    G64, x64 = down(G), orc.ckpt8_unpack(*stored8(x8))
    s64, add64 = None if scale is None else down(scale), None if more is None else down(more)
    out, around = room_for(d_out, d_in, torch.bfloat16 if bf16_out else torch.float32, pad)
    say("wgrad", tokens, d_out, d_in, scaled, add, bf16_out, pad)
    ah.adahop_ckpt8_wgrad(G, x8, col_scale=scale, add=more, Cout=out)
    want = orc.wgrad(G64, x64, s64, add64)
    bound = wgrad_bound(G64, x64, s64, tokens) + (0 if more is None else 2.0 ** -23 * (np.abs(want) + np.abs(add64))) + (BF16 * np.abs(want) if bf16_out else 0) + 1e-37
    off = np.abs(down(out) - want)
    assert np.all(off <= bound), f"{np.max(off / bound):.2f} times what is allowed"
    assert torch.all(around == 7)
    again = ah.adahop_ckpt8_wgrad(G, x8, col_scale=scale, add=more, c_bf16=bf16_out)
    assert torch.equal(again, out), "other bits in a second call"
    if more is not None and more.dtype == out.dtype:                # on top of what is there
        here = ah.adahop_ckpt8_wgrad(G, x8, col_scale=scale, add=more, Cout=more)
        assert torch.equal(here, out)


@pytest.mark.parametrize("tokens", [40, 130])
def test_wgrad_of_infinities_and_nan(ah, tokens):
    """They reach the elements whose sums they are in and no others, at the end of the tokens too."""
    rng = np.random.default_rng(3)
    d_out, d_in = 72, 96
    G = up(rng.normal(size=(tokens, d_out)))
    x = up(rng.normal(size=(tokens, d_in)))
    clean = ah.adahop_ckpt8_wgrad(G, ah.adahop_ckpt8_pack(x))
    G[tokens - 1, 5] = float("inf")
    x[tokens - 1, 7] = float("nan")
    x8 = ah.adahop_ckpt8_pack(x)
    say("wgrad with infinities", tokens)
    got = ah.adahop_ckpt8_wgrad(G, x8)
    assert bool(got[:, 7].isnan().all()) and not bool(got[5].isfinite().any())
    rest = torch.ones_like(got, dtype=torch.bool)
    rest[5], rest[:, 7] = False, False
    block = torch.zeros_like(rest)
    block[:, :32] = True                        # the last token's first block may have another scale without the NaN
    assert torch.equal(got[rest & ~block], clean[rest & ~block]) and bool(got[rest].isfinite().all())


# ---- no rows, other streams, graphs ----------------------------------------------------------------------------------------------------
def test_no_rows(ah):
    e = torch.empty(0, 96, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(96, dtype=torch.bfloat16, device="cuda")
    say("no rows")
    assert ah.adahop_ckpt8_pack(e)[1].shape == (0, 3)
    r = ah.adahop_block_norm(e, e, w_post=w, w_pre=w, gate=w, keep="ckpt8")
    assert r["h"].shape == (0, 96)
    assert ah.adahop_swiglu(e, e, keep8=True)["a"].shape == (0, 96)
    ah.adahop_swiglu_backward(e, e, e)
    b = ah.adahop_block_norm_backward(e, e, e, e, r["rstd_pre"], r["rstd_post"], w_post=w, w_pre=w, gate=w)
    assert all(float(b[n].float().abs().sum()) == 0 for n in ("d_w_post", "d_w_pre", "d_gate"))


def test_gate_rows_that_no_row_takes(ah):
    """Their gradient is zero."""
    x = torch.randn(10, 96, device="cuda").to(torch.bfloat16)
    gate = torch.ones(5, 96, dtype=torch.bfloat16, device="cuda")
    f = ah.adahop_block_norm(x, x, gate=gate, gate_rows=4, keep="stats")
    say("spare gate rows")
    b = ah.adahop_block_norm_backward(x, x, f["s"], x, f["rstd_pre"], f["rstd_post"], gate=gate, gate_rows=4)
    assert float(b["d_gate"][3:].float().abs().sum()) == 0 and bool((b["d_gate"][:3] != 0).any(1).all())


def everything(ah, x, y, d, w, G):
    f = ah.adahop_block_norm(x, y, w_post=w, w_pre=w, gate=w, keep="ckpt8")
    a = ah.adahop_swiglu(f["h"], y, keep8=True)
    a8 = ah.adahop_ckpt8_empty(*x.shape)
    da = ah.adahop_swiglu_backward(a["ckpt_g"], a["ckpt_u"], d, a=a8)
    b = ah.adahop_block_norm_backward(d, da["d_g"], f["ckpt_s"], f["ckpt_y"], f["rstd_pre"], f["rstd_post"], w_post=w, w_pre=w, gate=w)
    return [f["s"], f["h"], a["a"], da["d_u"], a8[0], b["d_x"], b["d_y"], b["d_w_post"], b["d_w_pre"], b["d_gate"], ah.adahop_ckpt8_wgrad(G, a8),
            ah.adahop_ckpt8_unpack(a8, col_scale=w)]


def operands(rows=513, cols=1048):
    gen = torch.Generator(device="cuda").manual_seed(9)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    return r(rows, cols), r(rows, cols), r(rows, cols), r(cols), r(rows, 136)


def test_on_another_stream(ah):
    args = operands()
    want = everything(ah, *args)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    say("another stream")
    with torch.cuda.stream(other):
        got = everything(ah, *args)
    other.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    x8 = ah.adahop_ckpt8_pack(args[0], stream=other)
    other.synchronize()
    assert torch.equal(x8[0], ah.adahop_ckpt8_pack(args[0])[0])


def test_from_a_graph(ah):
    """Captured once, replayed on new values with eager work between; every replay against the eager result."""
    args = operands()
    ah.adahop_prepare_device()
    everything(ah, *args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    say("graph")
    with torch.cuda.graph(graph):
        got = everything(ah, *args)
    for turn in range(3):
        for t in args[:3]:
            t.mul_(-0.5 if turn else 1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = everything(ah, *args)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), turn
