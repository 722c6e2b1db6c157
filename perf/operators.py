"""The training operators around a linear layer's products, as timed cases: a plain form of each in elementary torch
operations, and the calls of paper_2604_02525_amd.binding that compute the same.

  norm_fwd / norm_bwd      the norms after one block and before the next, with the block's gate and the residual scales:
                           s = alpha x + beta gate * w_post * yhat,  h = w_pre * shat, yhat and shat being y and s over their root
                           mean squares; and the gradients of x, y, both weights and the gate
  swiglu_fwd / swiglu_bwd  a = silu(g) u of a gated MLP, and its backward pass, which hands a back for the down projection
  pack / unpack            an activation to and from its 8-bit checkpoint
  wgrad                    G_W = G_Y^T X of a linear layer from X's 8-bit checkpoint

An 8-bit checkpoint holds E4M3 elements and one power-of-two scale (E8M0) for each 32 features of a token, the last ones of
an odd width fewer; as outputs they are tensors of these two 8-bit floating types.  Activations are N(0, 1) with 16 channels x 50, output
gradients N(0, 0.001) with 0.5 % of the token rows x 100, as everywhere in this repository.
"""
import math

import torch

own = False

WIDTHS = (2048, 4096, 8192)                     # hidden sizes of the library's configurations
FFN = (8192, 11008, 14336, 28672)               # and MLP widths
TOKENS = 16384
EPS = 1e-6


# ---- cases ------------------------------------------------------------------------------------------------------------

def _norm(kind, rows, cols, gate, keep, f32=False, name=None):
    """gate: none, vector (one per channel), sequence (one row per 4096 tokens), token.  keep: 8-bit checkpoints (forward:
    written, backward: read) in place of the tensors themselves.  f32: the residual stream and its gradient in 32 bits."""
    case = {"kind": kind, "rows": rows, "cols": cols, "gate": gate, "keep": keep, "f32": f32}
    return dict(case, name=name) if name else case


def _swiglu(kind, rows, cols, keep, f32=False, name=None):
    """forward: keep = g and u are also written in 8 bits; backward: keep = they are read in 8 bits and a is handed back
    in 8 bits, otherwise in bf16.  f32: g and u (forward) or a's gradient (backward) in 32 bits, as a product leaves them."""
    case = {"kind": kind, "rows": rows, "cols": cols, "keep": keep, "f32": f32}
    return dict(case, name=name) if name else case


def _wgrad(tokens, d_out, d_in, scaled, add, bf16_out, name=None):
    """scaled: times a norm's weight per input feature; add: on top of earlier micro-batches' gradient."""
    case = {"kind": "wgrad", "tokens": tokens, "d_out": d_out, "d_in": d_in, "scaled": scaled, "add": add, "bf16_out": bf16_out}
    return dict(case, name=name) if name else case


def _ckpt(kind, rows, cols, f32=False, name=None):
    case = {"kind": kind, "rows": rows, "cols": cols, "f32": f32}
    return dict(case, name=name) if name else case


def listed():
    return [
        # one token of a generation step between two blocks
        _norm("norm_fwd", 1, 4096, "vector", False, name="norm_fwd_1x4096"),
        # a training step's largest configuration, everything for the backward pass kept in 8 bits
        _norm("norm_fwd", 16384, 8192, "vector", True, name="norm_fwd_16384x8192_keep"),
        # a short ragged batch of an odd width, the residual stream in 32 bits, a gate for each token
        _norm("norm_bwd", 777, 4091, "token", False, f32=True, name="norm_bwd_777x4091_f32"),
        # the backward of the second one
        _norm("norm_bwd", 16384, 8192, "vector", True, name="norm_bwd_16384x8192_keep"),
        # the MLP of the LLaMA-7B-shaped configuration: forward, backward
        _swiglu("swiglu_fwd", 8192, 11008, True, name="swiglu_fwd_8192x11008_keep"),
        _swiglu("swiglu_bwd", 8192, 11008, True, name="swiglu_bwd_8192x11008_keep"),
        # a ragged batch of a width that is no multiple of anything, g and u at hand as they were, gradient in 32 bits
        _swiglu("swiglu_bwd", 301, 14333, False, f32=True, name="swiglu_bwd_301x14333_f32"),
        # the input of an output projection kept for the backward pass, and brought back for a product in other formats
        _ckpt("pack", 8192, 4096, name="pack_8192x4096"),
        _ckpt("unpack", 16384, 8192, name="unpack_16384x8192"),
        # a small layer's gradient over a ragged number of tokens
        _wgrad(1001, 2048, 2048, False, False, True, name="wgrad_1001_2048x2048"),
        # an attention projection fed by a norm, accumulated over micro-batches
        _wgrad(8192, 4096, 4096, True, True, False, name="wgrad_8192_4096x4096"),
        # the up projection of the largest configuration
        _wgrad(TOKENS, 28672, 8192, True, False, False, name="wgrad_16384_28672x8192"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("norm_fwd", "norm_bwd", "norm_bwd", "swiglu_fwd", "swiglu_bwd", "pack", "unpack", "wgrad", "wgrad"))
    odd = rng.random() < 0.3
    if kind == "wgrad":
        d_out, d_in = rng.choice(WIDTHS + FFN), rng.choice(WIDTHS)
        if odd:
            d_out, d_in = _log_int(rng, 64, 4096), _log_int(rng, 64, 4096)
        return _wgrad(_log_int(rng, 1, TOKENS), d_out, d_in, rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.3)
    rows = _log_int(rng, 1, TOKENS)
    if kind.startswith("norm"):
        cols = _log_int(rng, 64, 8192) if odd else rng.choice(WIDTHS)
        return _norm(kind, rows, cols, rng.choice(("none", "vector", "sequence", "token")), rng.random() < 0.6, rng.random() < 0.25)
    rows = min(rows, 8192)
    cols = _log_int(rng, 64, 11008) if odd else rng.choice(WIDTHS + (11008,))
    if kind.startswith("swiglu"):
        return _swiglu(kind, rows, cols, rng.random() < 0.6, rng.random() < 0.25)
    return _ckpt(kind, rows, cols, rng.random() < 0.25)


# ---- plain forms ------------------------------------------------------------------------------------------------------

def _by_32(v):
    """[rows, cols] as blocks of 32 features, the last one filled up with zeros."""
    rows, cols = v.shape
    return torch.nn.functional.pad(v, (0, -cols % 32)).view(rows, -1, 32)


def _pack(v):
    """v in 32 bits -> (E4M3 elements, E8M0 scales): scale = 2^(floor(log2 amax) - 8), to nearest even, saturating at 448."""
    b = _by_32(v)
    e = torch.frexp(b.abs().amax(2, keepdim=True)).exponent - 9
    e = torch.where(b.abs().amax(2, keepdim=True) > 0, e, torch.full_like(e, -127)).clamp(-127, 127)
    q = torch.ldexp(b, -e).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    scales = (e[:, :, 0] + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
    return q.view(v.shape[0], -1)[:, :v.shape[1]], scales


def _value(kept):
    """What a checkpoint stands for, in 32 bits."""
    codes, scales = kept
    return (_by_32(codes.float()) * scales.float()[:, :, None]).view(codes.shape[0], -1)[:, :codes.shape[1]]


def _gate_of(s):
    """The gate of every row, in 32 bits ([1, cols] where it is one for all)."""
    if s["gate"] is None:
        return None
    g = s["gate"].float()
    return g[None] if g.dim() == 1 else torch.repeat_interleave(g, s["gate_rows"], dim=0)[:s["rows"]]


def _norm_fwd(s):
    x, y, gate = s["x"].float(), s["y"].float(), _gate_of(s)
    r_post = torch.rsqrt((y * y).mean(1) + EPS)
    yhat = y * r_post[:, None]
    branch = yhat * s["w_post"].float()
    if gate is not None:
        branch = branch * gate
    z = s["alpha"] * x + s["beta"] * branch
    r_pre = torch.rsqrt((z * z).mean(1) + EPS)
    shat = z * r_pre[:, None]
    return z, shat * s["w_pre"].float(), yhat, shat, r_post, r_pre


def _norm_fwd_out(s):
    z, h, yhat, shat, r_post, r_pre = _norm_fwd(s)
    out = {"s": z.to(s["x"].dtype), "h": h.to(torch.bfloat16)}
    if s["keep"]:
        out |= {"ckpt_y": _pack(yhat), "ckpt_s": _pack(shat), "rstd_post": r_post, "rstd_pre": r_pre}
    return out


def _norm_bwd_out(s):
    if s["keep"]:
        yhat, shat = _value(s["ckpt_y"]), _value(s["ckpt_s"])
    else:
        yhat, shat = s["y"].float() * s["rstd_post"][:, None], s["s"].float() * s["rstd_pre"][:, None]
    w_post, w_pre, gate, dh = s["w_post"].float(), s["w_pre"].float(), _gate_of(s), s["d_h"].float()
    t = dh * w_pre
    d = s["d_s"].float() + s["rstd_pre"][:, None] * (t - shat * (t * shat).mean(1, keepdim=True))
    u = s["beta"] * d
    v = u * w_post if gate is None else u * w_post * gate
    dy = s["rstd_post"][:, None] * (v - yhat * (v * yhat).mean(1, keepdim=True))
    uy = u * yhat
    out = {"d_x": (s["alpha"] * d).to(s["d_s"].dtype), "d_y": dy.to(torch.bfloat16), "d_w_pre": (dh * shat).sum(0),
           "d_w_post": (uy if gate is None else uy * gate).sum(0)}
    if gate is not None:
        dg = uy * w_post
        if s["gate"].dim() == 1:
            dg = dg.sum(0)
        else:
            n = s["gate"].shape[0]
            dg = torch.nn.functional.pad(dg, (0, 0, 0, n * s["gate_rows"] - dg.shape[0])).view(n, s["gate_rows"], -1).sum(1)
        out["d_gate"] = dg.to(s["gate"].dtype)
    return out


def _swiglu_fwd_out(s):
    g, u = s["g"].float(), s["u"].float()
    out = {"a": (g * torch.sigmoid(g) * u).to(torch.bfloat16)}
    if s["keep"]:
        out |= {"ckpt_g": _pack(g), "ckpt_u": _pack(u)}
    return out


def _swiglu_bwd_out(s):
    g, u = (_value(s["ckpt_g"]), _value(s["ckpt_u"])) if s["keep"] else (s["g"].float(), s["u"].float())
    da, sig = s["d_a"].float(), torch.sigmoid(g)
    silu = g * sig
    a = silu * u
    return {"d_g": (da * u * (sig + silu * (1.0 - sig))).to(torch.bfloat16), "d_u": (da * silu).to(torch.bfloat16),
            "a": _pack(a) if s["keep"] else a.to(torch.bfloat16)}


def _wgrad_out(s):
    c = s["G"].float().t() @ _value(s["x8"])
    if s["col_scale"] is not None:
        c = c * s["col_scale"].float()
    if s["add"] is not None:
        c = c + s["add"].float()
    return {"C": c.to(s["C"].dtype)}


# ---- inputs -----------------------------------------------------------------------------------------------------------

def _rand(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std)


def _activation(gen, rows, cols):
    x = _rand(gen, rows, cols)
    x[:, torch.randperm(cols, generator=gen, device="cuda")[:16]] *= 50.0
    return x


def _gradient(gen, rows, cols):
    x = _rand(gen, rows, cols, std=1e-3)
    x[torch.randperm(rows, generator=gen, device="cuda")[:int(math.ceil(0.005 * rows))]] *= 100.0
    return x


def _weight(gen, cols):
    return _rand(gen, cols, std=0.2).add_(1.0).to(torch.bfloat16)


def _rows_of(cols, rows, dtype, multiple=1):
    """An empty [rows, cols] whose rows begin at multiples of `multiple` elements."""
    return torch.empty(rows, -(-cols // multiple) * multiple, dtype=dtype, device="cuda")[:, :cols]


def _kept(v):
    """A checkpoint as a program holds it: rows of codes at multiples of 16 bytes."""
    codes, scales = _pack(v)
    held = _rows_of(codes.shape[1], codes.shape[0], torch.uint8, 16)
    held.copy_(codes.contiguous().view(torch.uint8))
    return held.view(torch.float8_e4m3fn), scales


def _room(rows, cols):
    """Where a checkpoint is written."""
    return (_rows_of(cols, rows, torch.uint8, 16), torch.empty(rows, -(-cols // 32), dtype=torch.uint8, device="cuda"))


def _prepare_norm(gen, case):
    rows, cols, stream = case["rows"], case["cols"], torch.float32 if case["f32"] else torch.bfloat16
    s = {"rows": rows, "keep": case["keep"], "alpha": 1.0, "beta": 0.5, "gate": None, "gate_rows": 1,
         "x": _activation(gen, rows, cols).to(stream), "y": _activation(gen, rows, cols).to(torch.bfloat16),
         "w_post": _weight(gen, cols), "w_pre": _weight(gen, cols)}
    if case["gate"] == "vector":
        s["gate"] = _weight(gen, cols)
    elif case["gate"] != "none":
        s["gate_rows"] = 1 if case["gate"] == "token" else 4096
        s["gate"] = _rand(gen, -(-rows // s["gate_rows"]), cols).to(torch.bfloat16)
    empty = lambda dtype: torch.empty(rows, cols, dtype=dtype, device="cuda")  # noqa: E731
    if case["kind"] == "norm_fwd":
        s["out"] = {"s": empty(stream), "h": empty(torch.bfloat16)}
        if case["keep"]:
            s["out"] |= {"ckpt_y": _room(rows, cols), "ckpt_s": _room(rows, cols)}
            s["out"] |= {k: torch.empty(rows, dtype=torch.float32, device="cuda") for k in ("rstd_post", "rstd_pre")}
        return s
    z, _, yhat, shat, s["rstd_post"], s["rstd_pre"] = _norm_fwd(s)
    if case["keep"]:
        s["ckpt_y"], s["ckpt_s"] = _kept(yhat), _kept(shat)
        del s["y"]
    else:
        s["s"] = z.to(stream)
    del s["x"]
    s["d_s"], s["d_h"] = _gradient(gen, rows, cols).to(stream), _gradient(gen, rows, cols).to(torch.bfloat16)
    s["out"] = {"d_x": empty(stream), "d_y": empty(torch.bfloat16),
                "d_w_pre": torch.empty(cols, dtype=torch.float32, device="cuda"), "d_w_post": torch.empty(cols, dtype=torch.float32, device="cuda"),
                "d_gate": None if s["gate"] is None else torch.empty_like(s["gate"])}
    return s


def _prepare_swiglu(gen, case):
    rows, cols = case["rows"], case["cols"]
    wide = torch.float32 if case["f32"] else torch.bfloat16
    both = torch.cat((_rand(gen, rows, cols, std=2.0), _activation(gen, rows, cols)), 1)        # one product's [g | u]
    empty = lambda: torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    s = {"keep": case["keep"]}
    if case["kind"] == "swiglu_fwd":
        both = both.to(wide)
        s["out"] = {"a": empty()}
        if case["keep"]:
            s["out"] |= {"ckpt_g": _room(rows, cols), "ckpt_u": _room(rows, cols)}
        return s | {"g": both[:, :cols], "u": both[:, cols:]}
    if case["keep"]:
        s |= {"ckpt_g": _kept(both[:, :cols].to(torch.bfloat16).float()), "ckpt_u": _kept(both[:, cols:].to(torch.bfloat16).float())}
    else:
        both = both.to(torch.bfloat16)
        s |= {"g": both[:, :cols], "u": both[:, cols:]}
    s["d_a"] = _gradient(gen, rows, cols).to(wide)
    d_both = torch.empty(rows, 2 * cols, dtype=torch.bfloat16, device="cuda")
    s["out"] = {"d_g": d_both[:, :cols], "d_u": d_both[:, cols:], "a": _room(rows, cols) if case["keep"] else empty()}
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    if kind.startswith("norm"):
        return {"kind": kind} | _prepare_norm(gen, case)
    if kind.startswith("swiglu"):
        return {"kind": kind} | _prepare_swiglu(gen, case)
    if kind == "wgrad":
        T, N, D = case["tokens"], case["d_out"], case["d_in"]
        G = _rows_of(N, T, torch.bfloat16, 8)
        G.copy_(_gradient(gen, T, N))
        return {"kind": kind, "G": G, "x8": _kept(_activation(gen, T, D).to(torch.bfloat16).float()),
                "col_scale": _weight(gen, D) if case["scaled"] else None, "add": _rand(gen, N, D, std=1e-2) if case["add"] else None,
                "C": torch.empty(N, D, dtype=torch.bfloat16 if case["bf16_out"] else torch.float32, device="cuda")}
    x = _activation(gen, case["rows"], case["cols"]).to(torch.float32 if case["f32"] and kind == "pack" else torch.bfloat16)
    if kind == "pack":
        return {"kind": kind, "x": x, "out": _room(case["rows"], case["cols"])}
    return {"kind": kind, "x8": _kept(x.float()),
            "out": torch.empty(case["rows"], case["cols"], dtype=torch.float32 if case["f32"] else torch.bfloat16, device="cuda")}


# ---- one pass ---------------------------------------------------------------------------------------------------------

def _floats(kept):
    """A checkpoint's bytes as what they are."""
    return kept[0].view(torch.float8_e4m3fn), kept[1].view(torch.float8_e8m0fnu)


def _bytes(kept):
    return kept[0].view(torch.uint8), kept[1].view(torch.uint8)


def _run_own(s):
    from paper_2604_02525_amd import binding as ah
    kind, out = s["kind"], s.get("out")
    if kind == "norm_fwd":
        r = ah.adahop_block_norm(s["x"], s["y"], w_post=s["w_post"], w_pre=s["w_pre"], gate=s["gate"], gate_rows=s["gate_rows"],
                                 residual_scale=s["alpha"], branch_scale=s["beta"], eps=EPS, **out)
        got = {"s": r["s"], "h": r["h"]}
        if s["keep"]:
            got |= {"ckpt_y": _floats(r["ckpt_y"]), "ckpt_s": _floats(r["ckpt_s"]), "rstd_post": r["rstd_post"], "rstd_pre": r["rstd_pre"]}
        return got
    if kind == "norm_bwd":
        y, z = (_bytes(s["ckpt_y"]), _bytes(s["ckpt_s"])) if s["keep"] else (s["y"], s["s"])
        r = ah.adahop_block_norm_backward(s["d_s"], s["d_h"], z, y, s["rstd_pre"], s["rstd_post"], w_post=s["w_post"], w_pre=s["w_pre"],
                                          gate=s["gate"], gate_rows=s["gate_rows"], residual_scale=s["alpha"], branch_scale=s["beta"], **out)
        return {k: r[k] for k in ("d_x", "d_y", "d_w_pre", "d_w_post") + (("d_gate",) if s["gate"] is not None else ())}
    if kind == "swiglu_fwd":
        r = ah.adahop_swiglu(s["g"], s["u"], **out)
        return {"a": r["a"]} | ({"ckpt_g": _floats(r["ckpt_g"]), "ckpt_u": _floats(r["ckpt_u"])} if s["keep"] else {})
    if kind == "swiglu_bwd":
        g, u = (_bytes(s["ckpt_g"]), _bytes(s["ckpt_u"])) if s["keep"] else (s["g"], s["u"])
        r = ah.adahop_swiglu_backward(g, u, s["d_a"], **out)
        return {"d_g": r["d_g"], "d_u": r["d_u"], "a": _floats(r["a"]) if s["keep"] else r["a"]}
    if kind == "pack":
        return _floats(ah.adahop_ckpt8_pack(s["x"], out=out))
    if kind == "unpack":
        return ah.adahop_ckpt8_unpack(_bytes(s["x8"]), out=out)
    return {"C": ah.adahop_ckpt8_wgrad(s["G"], _bytes(s["x8"]), col_scale=s["col_scale"], add=s["add"], Cout=s["C"])}


def run(state):
    if own:
        return _run_own(state)
    kind = state["kind"]
    if kind == "norm_fwd":
        return _norm_fwd_out(state)
    if kind == "norm_bwd":
        return _norm_bwd_out(state)
    if kind == "swiglu_fwd":
        return _swiglu_fwd_out(state)
    if kind == "swiglu_bwd":
        return _swiglu_bwd_out(state)
    if kind == "pack":
        return _pack(state["x"].float())
    if kind == "unpack":
        return _value(state["x8"]).to(state["out"].dtype)
    return _wgrad_out(state)


def work(case):
    kind, kept = case["kind"], 1 + 1 / 32
    if kind == "wgrad":
        T, N, D = float(case["tokens"]), float(case["d_out"]), float(case["d_in"])
        return {"bytes": 2 * T * N + kept * T * D + (2 if case["bf16_out"] else 4) * N * D + (4 * N * D if case["add"] else 0) + (2 * D if case["scaled"] else 0),
                "flops": 2 * T * N * D}
    rows, cols = float(case["rows"]), float(case["cols"])
    n, wide = rows * cols, 4 if case["f32"] else 2
    if kind == "pack":
        return {"bytes": (wide + kept) * n, "flops": 0.0}
    if kind == "unpack":
        return {"bytes": (wide + kept) * n, "flops": 0.0}
    if kind == "swiglu_fwd":
        return {"bytes": (2 * wide + 2 + (2 * kept if case["keep"] else 0)) * n, "flops": 8 * n}
    if kind == "swiglu_bwd":
        return {"bytes": (wide + 4 + (3 * kept if case["keep"] else 6)) * n, "flops": 14 * n}
    gates = {"none": 0.0, "vector": cols, "sequence": cols * math.ceil(rows / 4096), "token": n}[case["gate"]]
    if kind == "norm_fwd":
        return {"bytes": (2 * wide + 4 + (2 * kept if case["keep"] else 0)) * n + 2 * gates + 4 * cols + (8 * rows if case["keep"] else 0), "flops": 10 * n}
    return {"bytes": (2 * wide + 4 + (2 * kept if case["keep"] else wide + 2)) * n + 4 * gates + 12 * cols + 8 * rows, "flops": 22 * n}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------

def _unkeep64(codes, scales):
    each = torch.pow(2.0, scales.view(torch.uint8).double() - 127.0).repeat_interleave(32, dim=1)
    return codes.double() * each[:, :codes.shape[1]]


def _keep64(v):
    """The elements and scales that v's checkpoint has, as numbers."""
    rows, cols = v.shape
    blocks = (cols + 31) // 32
    amax = torch.zeros(rows, blocks, dtype=torch.float64, device=v.device)
    amax.scatter_reduce_(1, (torch.arange(cols, device=v.device) // 32).expand(rows, cols), v.abs(), "amax")
    scale = torch.where(amax > 0, torch.exp2(torch.floor(torch.log2(amax.clamp_min(1e-300))) - 8), torch.full_like(amax, 2.0 ** -127)).clamp(2.0 ** -127, 2.0 ** 127)
    q = (v / scale.repeat_interleave(32, dim=1)[:, :cols])
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp_min(2.0 ** -6))) - 3)        # three bits behind the leading one, 2^-9 at least
    return (torch.round(q / step) * step).clamp(-448.0, 448.0), scale


def _gate64(s):
    if s["gate"] is None:
        return torch.ones(1, 1, dtype=torch.float64, device="cuda")
    g = s["gate"].double()
    return g.view(1, -1) if g.dim() == 1 else g[torch.arange(s["rows"], device="cuda") // s["gate_rows"]]


def _exact_norm_fwd(s):
    y = s["y"].double()
    r_post = (y.square().sum(1) / y.shape[1] + EPS).pow(-0.5)
    yhat = y * r_post[:, None]
    z = s["alpha"] * s["x"].double() + (s["beta"] * s["w_post"].double()) * _gate64(s) * yhat
    r_pre = (z.square().sum(1) / z.shape[1] + EPS).pow(-0.5)
    shat = z * r_pre[:, None]
    out = {"s": z, "h": shat * s["w_pre"].double()}
    if s["keep"]:
        out |= {"ckpt_y": _keep64(yhat), "ckpt_s": _keep64(shat), "rstd_post": r_post, "rstd_pre": r_pre}
    return out


def _exact_norm_bwd(s):
    r_post, r_pre = s["rstd_post"].double()[:, None], s["rstd_pre"].double()[:, None]
    if s["keep"]:
        yhat, shat = _unkeep64(*s["ckpt_y"]), _unkeep64(*s["ckpt_s"])
    else:
        yhat, shat = s["y"].double() * r_post, s["s"].double() * r_pre
    cols = yhat.shape[1]
    through = lambda grad, unit, r: r * (grad - unit * ((grad * unit).sum(1, keepdim=True) / cols))  # noqa: E731
    d_h, gate = s["d_h"].double(), _gate64(s)
    d = s["d_s"].double() + through(d_h * s["w_pre"].double(), shat, r_pre)
    d_branch = s["beta"] * d                                # of gate * w_post * yhat
    w_post = s["w_post"].double()
    out = {"d_x": s["alpha"] * d, "d_y": through(d_branch * (gate * w_post), yhat, r_post), "d_w_pre": torch.sum(d_h * shat, 0),
           "d_w_post": torch.sum(d_branch * gate * yhat, 0)}
    if s["gate"] is not None:
        per_row = d_branch * yhat * w_post
        if s["gate"].dim() == 1:
            out["d_gate"] = per_row.sum(0)
        else:
            at = torch.arange(s["rows"], device="cuda") // s["gate_rows"]
            out["d_gate"] = torch.zeros(s["gate"].shape, dtype=torch.float64, device="cuda").index_add_(0, at, per_row)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm_fwd":
        return _exact_norm_fwd(s)
    if kind == "norm_bwd":
        return _exact_norm_bwd(s)
    if kind == "swiglu_fwd":
        g, u = s["g"].double(), s["u"].double()
        out = {"a": g / (1 + torch.exp(-g)) * u}
        return out | ({"ckpt_g": _keep64(g), "ckpt_u": _keep64(u)} if s["keep"] else {})
    if kind == "swiglu_bwd":
        g, u = (_unkeep64(*s["ckpt_g"]), _unkeep64(*s["ckpt_u"])) if s["keep"] else (s["g"].double(), s["u"].double())
        e, d_a = 1 / (1 + torch.exp(-g)), s["d_a"].double()
        a = g * e * u
        return {"d_g": d_a * u * e * (1 + g * (1 - e)), "d_u": d_a * g * e, "a": _keep64(a) if s["keep"] else a}
    if kind == "pack":
        return _keep64(s["x"].double())
    if kind == "unpack":
        return _unkeep64(*s["x8"])
    c = torch.matmul(s["G"].double().t().contiguous(), _unkeep64(*s["x8"]))
    c = c if s["col_scale"] is None else c * s["col_scale"].double()[None]
    return {"C": c if s["add"] is None else c + s["add"].double()}
