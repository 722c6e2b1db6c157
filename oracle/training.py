"""Plain 64-bit definitions of the training operators around the products (block norm, gated activation, 8-bit checkpoints, weight
gradient from one).  numpy only, nothing shared with the library."""
import numpy as np

F64 = np.float64


# ---- 8-bit checkpoints: E4M3 elements, one power of two per 32 columns -----------------------------------------------------
def e4m3_table():
    """Value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; S.1111.111 is NaN, no infinity."""
    v = np.empty(256, F64)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        v[c] = np.nan if c & 127 == 127 else -x if c & 128 else x
    return v


E4M3 = e4m3_table()


def e4m3_encode(q):
    """To nearest, ties to the even code, saturating; NaN for what is not finite.  q: float64."""
    mags = E4M3[:127]
    a = np.abs(q)
    finite = np.isfinite(a)
    a = np.where(finite, np.minimum(a, 448.0), 0.0)
    hi = np.searchsorted(mags, a, side="left")
    lo = np.maximum(hi - 1, 0)
    down, up = a - mags[lo], mags[hi] - a
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    code = np.where(finite, code, 127)
    return (code | np.where(np.signbit(q), 128, 0)).astype(np.uint8)


def ckpt8_pack(x):
    """(codes [rows, cols], scales [rows, ceil(cols / 32)])"""
    x = np.asarray(x, F64)
    rows, cols = x.shape
    blocks = -(-cols // 32)
    scales = np.zeros((rows, blocks), np.uint8)
    codes = np.zeros((rows, cols), np.uint8)
    for b in range(blocks):
        part = x[:, 32 * b:32 * b + 32]
        amax = np.max(np.where(np.isfinite(part), np.abs(part), 0.0), axis=1)
        e = np.where(amax > 0, np.frexp(np.where(amax > 0, amax, 1.0))[1] - 1 - 8, -127)
        scales[:, b] = np.maximum(e + 127, 0)
        codes[:, 32 * b:32 * b + 32] = e4m3_encode(part * np.exp2(127.0 - scales[:, b].astype(F64))[:, None])
    return codes, scales


def ckpt8_unpack(codes, scales):
    value = np.where(scales == 255, np.nan, np.exp2(scales.astype(F64) - 127.0))        # E8M0: 255 is NaN
    return E4M3[codes] * np.repeat(value, 32, axis=1)[:, :codes.shape[1]]


# ---- gated activation ------------------------------------------------------------------------------------------------------
def _sigmoid(g):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-g))


def swiglu(g, u):
    return g * _sigmoid(g) * u


def swiglu_backward(g, u, d_a):
    s = _sigmoid(g)
    return d_a * u * (s + g * s * (1.0 - s)), d_a * g * s


# ---- block norm ------------------------------------------------------------------------------------------------------------
def gate_of_rows(gate, gate_rows, rows):
    """The gate of every row: ones, a vector for all, or each of its rows for gate_rows rows."""
    if gate is None:
        return np.ones((1, 1))
    return gate[None] if gate.ndim == 1 else gate[np.arange(rows) // gate_rows]


def block_norm(x, y, w_post, w_pre, gate=None, gate_rows=1, alpha=1.0, beta=1.0, eps=1e-6, post_norm=True):
    """dict(s, h, yhat, shat, r_y, r_s); x or y may be None."""
    some = y if x is None else x
    rows, cols = some.shape
    one = np.ones(cols)
    yhat, r_y = None, None
    s = np.zeros((rows, cols)) if x is None else alpha * x
    if y is not None:
        r_y = 1.0 / np.sqrt((y ** 2).mean(1) + eps) if post_norm else np.ones(rows)
        yhat = y * r_y[:, None]
        s = s + beta * gate_of_rows(gate, gate_rows, rows) * (one if w_post is None else w_post) * yhat
    r_s = 1.0 / np.sqrt((s ** 2).mean(1) + eps)
    shat = s * r_s[:, None]
    return dict(s=s, h=shat * (one if w_pre is None else w_pre), yhat=yhat, shat=shat, r_y=r_y, r_s=r_s)


def block_norm_backward(d_s, d_h, shat, yhat, r_s, r_y, w_post, w_pre, gate=None, gate_rows=1, alpha=1.0, beta=1.0, post_norm=True):
    """Gradients from those of s and h (None: zero), and what the rounding of each may be measured by (`mag`: the sums of the
    magnitudes of what is added)."""
    rows, cols = (d_s if d_h is None else d_h).shape
    one = np.ones(cols)
    w_post, w_pre = one if w_post is None else w_post, one if w_pre is None else w_pre
    d_s = np.zeros((rows, cols)) if d_s is None else d_s
    out, mag = {}, {}
    if d_h is not None:
        t = w_pre * d_h
        r = r_s[:, None]
        d = d_s + r * (t - shat * (t * shat).mean(1, keepdims=True))
        m = np.abs(d_s) + r * (np.abs(t) + np.abs(shat) * np.abs(t * shat).mean(1, keepdims=True))
        out["d_w_pre"], mag["d_w_pre"] = (d_h * shat).sum(0), np.abs(d_h * shat).sum(0)
    else:
        d, m = d_s, np.abs(d_s)
    out["d_x"], mag["d_x"] = alpha * d, abs(alpha) * m
    if yhat is None:
        return out, mag
    g = gate_of_rows(gate, gate_rows, rows)
    q = beta * g * w_post
    if post_norm:
        r = r_y[:, None]
        out["d_y"] = r * (q * d - yhat * (q * d * yhat).mean(1, keepdims=True))
        mag["d_y"] = r * (np.abs(q) * m + np.abs(yhat) * (np.abs(q) * m * np.abs(yhat)).mean(1, keepdims=True))
    else:
        out["d_y"], mag["d_y"] = q * d, np.abs(q) * m
    out["d_w_post"], mag["d_w_post"] = (beta * g * d * yhat).sum(0), (np.abs(beta * g) * m * np.abs(yhat)).sum(0)
    if gate is not None:
        dg, mg = beta * w_post * d * yhat, np.abs(beta * w_post) * m * np.abs(yhat)
        if gate.ndim == 1:
            out["d_gate"], mag["d_gate"] = dg.sum(0), mg.sum(0)
        else:
            out["d_gate"], mag["d_gate"] = np.zeros(gate.shape), np.zeros(gate.shape)
            np.add.at(out["d_gate"], np.arange(rows) // gate_rows, dg)
            np.add.at(mag["d_gate"], np.arange(rows) // gate_rows, mg)
    return out, mag


# ---- weight gradient -------------------------------------------------------------------------------------------------------
def wgrad(G, x, col_scale=None, add=None):
    c = G.T @ x
    c = c if col_scale is None else c * col_scale
    return c if add is None else c + add
