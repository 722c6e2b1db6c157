"""Plain 64-bit definitions of what a training step does behind the last block: softmax cross entropy over a vocabulary with its gradients, and
updates of weights by Newton-Schulz products.  numpy only, nothing shared with the library."""
import numpy as np

F64 = np.float64
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)


# ---- loss ---------------------------------------------------------------------------------------------------------------------
def logits(h, w, logit_scale=1.0):
    return logit_scale * (np.asarray(h, F64) @ np.asarray(w, F64).T)


def linear_ce(h, w, targets, logit_scale=1.0, z_loss=0.0):
    """(loss, lse)"""
    z = logits(h, w, logit_scale)
    top = z.max(axis=1)
    lse = top + np.log(np.exp(z - top[:, None]).sum(axis=1))
    loss = np.zeros(len(targets))
    for t, y in enumerate(targets):
        if y >= z.shape[1]:
            loss[t] = np.nan
        elif y >= 0:
            loss[t] = lse[t] - z[t, y] + z_loss * lse[t] ** 2
    return loss, lse


def linear_ce_dz(h, w, targets, lse, d_loss, logit_scale=1.0, z_loss=0.0):
    """Gradient of the products of h and w (of the logits before their scale)."""
    p = np.exp(logits(h, w, logit_scale) - lse[:, None]) * (1.0 + 2.0 * z_loss * lse)[:, None]
    for t, y in enumerate(targets):
        if y >= 0:
            p[t, y] -= 1.0
    gain = np.where(np.asarray(targets) >= 0, d_loss * logit_scale, 0.0)
    return p * gain[:, None]


def linear_ce_backward(h, w, targets, lse, d_loss, logit_scale=1.0, z_loss=0.0):
    """(d_h, d_w)"""
    dz = linear_ce_dz(h, w, targets, lse, d_loss, logit_scale, z_loss)
    return dz @ np.asarray(w, F64), dz.T @ np.asarray(h, F64)


# ---- updates --------------------------------------------------------------------------------------------------------------------
def newton_schulz(u, steps=5, coefficients=NEWTON_SCHULZ, eps=1e-7):
    a, b, c = coefficients
    x = np.asarray(u, F64)
    x = x / (np.sqrt((x * x).sum()) + eps)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T
    for _ in range(steps):
        g = x @ x.T
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.T if tall else x


def _fp16(x, scale):
    return (x * scale).astype(np.float16).astype(F64) / scale


def newton_schulz_held(u, steps=5, coefficients=NEWTON_SCHULZ, eps=1e-7, split=False):
    """The same with the roundings of a form that holds X in 32 bits and lets fp16 numbers into the products, the diagonals apart; split: X as two of them.
    (A form whose diagonals, too, take X as rounded in the first steps loses less where X has few directions, and up to twice as much where it has all.)"""
    a, b, c = coefficients
    x = np.asarray(u, F64)
    x = x / (np.sqrt((x * x).sum()) + eps)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.T
    for _ in range(steps):
        x = x.astype(np.float32).astype(F64)
        high = _fp16(x, 2.0 ** 12)
        low = _fp16(x - high, 2.0 ** 12) if split else 0.0 * x
        g = high @ high.T + high @ low.T + low @ high.T
        d = np.diag(g).copy()
        o = _fp16(g - np.diag(d), 2.0 ** 12)
        oo = o @ o
        p = b * o + c * ((d[:, None] + d[None, :]) * o + oo)
        diagonal = a + b * d + c * (d * d + np.diag(oo))
        p = _fp16(p - np.diag(np.diag(p)), 2.0 ** 10)
        x = diagonal[:, None] * x + p @ (high + low)
    return x.T if tall else x


def momentum(m, g, mu, nesterov):
    """(m', U)"""
    m = mu * np.asarray(m, F64) + np.asarray(g, F64)
    return m, np.asarray(g, F64) + mu * m if nesterov else m
