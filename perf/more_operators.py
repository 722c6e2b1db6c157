"""The two ends of a training step that lie behind the last block, as timed cases: the loss over a vocabulary with its gradients, and the
update of a weight matrix.  A plain form of each in elementary torch operations, and the calls of paper_2604_02525_amd.binding that compute
the same.

  ce_fwd / ce_bwd   softmax cross entropy of z = logit_scale h W^T against one target per token, the logits never kept:
                    loss = lse - z[target] + z_loss lse^2,  lse = log sum exp z;  and the gradients of h and W
  orth              a matrix orthogonalised by Newton-Schulz products:  X = G / (|G| + eps),  then X <- a X + (b A + c A^2) X, A = X X^T
  muon              one update of a weight: momentum, orthogonalised direction, weight decay, the masters and their bf16 copy

Activations are N(0, 1) with 16 channels x 50 and weights N(0, 0.02), as everywhere in this repository; a weight's gradient is
a product of token gradients and activations, so a few directions of it are strong.
"""
import math

import torch

own = False

WIDTHS = (2048, 4096, 8192)                     # hidden sizes of the library's configurations
TOKENS = 16384
LARGEST = 16384 * 8192 * 65536                  # tokens x width x vocabulary of the largest loss
IGNORED = -100
STEPS, COEFFICIENTS, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
MU = 0.95


# ---- cases ------------------------------------------------------------------------------------------------------------

def _ce(kind, tokens, dim, vocab, ignored=0.0, logit_scale=1.0, z_loss=0.0, name=None):
    """ignored: the share of tokens without a target (padding, prompts)."""
    case = {"kind": kind, "tokens": tokens, "dim": dim, "vocab": vocab, "ignored": ignored, "logit_scale": logit_scale, "z_loss": z_loss}
    return dict(case, name=name) if name else case


def _orth(rows, cols, f32=False, name=None):
    """f32: the matrix in 32 bits, else in bf16; the result is bf16."""
    case = {"kind": "orth", "rows": rows, "cols": cols, "f32": f32}
    return dict(case, name=name) if name else case


def _muon(rows, cols, f32=True, nesterov=True, decay=0.0, name=None):
    """f32: the gradient in 32 bits, else in bf16."""
    case = {"kind": "muon", "rows": rows, "cols": cols, "f32": f32, "nesterov": nesterov, "decay": decay}
    return dict(case, name=name) if name else case


def listed():
    return [
        # the likelihood of one token of a generation step
        _ce("ce_fwd", 1, 4096, 32000, name="ce_fwd_1x4096_32000"),
        # held-out loss of a ragged batch of packed documents, prompts without targets, an odd vocabulary
        _ce("ce_fwd", 1003, 2048, 50021, ignored=0.3, name="ce_fwd_1003x2048_50021"),
        # the loss of a training step: four sequences of 2048 tokens
        _ce("ce_fwd", 8192, 4096, 32000, ignored=0.01, name="ce_fwd_8192x4096_32000"),
        # gradients of a short ragged batch, logits scaled and kept near zero
        _ce("ce_bwd", 777, 2056, 30011, ignored=0.1, logit_scale=0.5, z_loss=1e-4, name="ce_bwd_777x2056_30011"),
        # the backward pass of the training step
        _ce("ce_bwd", 8192, 4096, 32000, ignored=0.01, name="ce_bwd_8192x4096_32000"),
        # the largest configuration's tokens and width, a large vocabulary
        _ce("ce_bwd", 16384, 8192, 65536, z_loss=1e-4, name="ce_bwd_16384x8192_65536"),
        # a small matrix (an adapter, one head's projection): latency
        _orth(256, 256, name="orth_256x256"),
        # a matrix of odd sizes, the gradient in 32 bits
        _orth(1001, 2333, f32=True, name="orth_1001x2333_f32"),
        # an attention projection
        _orth(4096, 4096, name="orth_4096x4096"),
        # an output projection of a small model, the gradient as a bf16 product leaves it
        _muon(2048, 2048, f32=False, decay=0.1, name="muon_2048x2048"),
        # the down projection of the LLaMA-7B-shaped configuration
        _muon(4096, 11008, decay=0.1, name="muon_4096x11008"),
        # the up projection of the largest configuration: a tall matrix
        _muon(28672, 8192, decay=0.1, name="muon_28672x8192"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("ce_fwd", "ce_bwd", "ce_bwd", "orth", "orth", "muon", "muon"))
    odd = rng.random() < 0.4
    if kind.startswith("ce"):
        tokens, vocab = _log_int(rng, 1, TOKENS), rng.choice((32000, 65536, 131072))
        dim = rng.choice(WIDTHS)
        if odd:
            dim, vocab = _log_int(rng, 64, 8192), _log_int(rng, 256, 131072)
        tokens = max(1, min(tokens, LARGEST // (dim * vocab)))
        return _ce(kind, tokens, dim, vocab, rng.choice((0.0, 0.01, 0.3)), rng.choice((1.0, 1.0, 0.5)), rng.choice((0.0, 1e-4)))
    rows, cols = 64 * _log_int(rng, 4, 128), 64 * _log_int(rng, 4, 448)
    if rng.random() < 0.5:
        rows, cols = cols, rows
    if odd:
        rows, cols = _log_int(rng, 48, 6000), _log_int(rng, 48, 6000)
    if kind == "orth":
        return _orth(rows, cols, rng.random() < 0.5)
    return _muon(rows, cols, rng.random() < 0.6, rng.random() < 0.7, rng.choice((0.0, 0.1)))


# ---- plain forms ------------------------------------------------------------------------------------------------------

def _logits(s):
    return (s["h"].float() @ s["w"].float().t()) * s["logit_scale"]


def _ce_fwd_out(s):
    z = _logits(s)
    top = z.amax(1)
    lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    there = s["targets"] >= 0
    at = z.gather(1, s["targets"].clamp(min=0)[:, None])[:, 0]
    return {"loss": torch.where(there, lse - at + s["z_loss"] * lse * lse, torch.zeros_like(lse)), "lse": lse}


def _ce_bwd_out(s):
    z, lse = _logits(s), s["lse"]
    there = s["targets"] >= 0
    dz = torch.exp(z - lse[:, None])
    dz *= (1.0 + 2.0 * s["z_loss"] * lse)[:, None]
    dz.scatter_add_(1, s["targets"].clamp(min=0)[:, None], torch.full_like(lse, -1.0)[:, None])
    dz *= torch.where(there, s["d_loss"] * s["logit_scale"], torch.zeros_like(lse))[:, None]
    return {"d_h": (dz @ s["w"].float()).to(torch.bfloat16), "d_w": (dz.t() @ s["h"].float()).to(torch.bfloat16)}


def _newton_schulz(x):
    """x in 32 bits."""
    a, b, c = COEFFICIENTS
    x = x / (torch.sqrt((x.double() * x.double()).sum()).float() + EPS)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    x = x.contiguous()
    for _ in range(STEPS):  # the method's own steps
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if tall else x


def _orth_out(s):
    return {"out": _newton_schulz(s["g"].float()).to(torch.bfloat16)}


def _muon_out(s):
    g = s["g"].float()
    m = MU * s["momentum"] + g
    o = _newton_schulz(g + MU * m if s["nesterov"] else m)
    w = (1.0 - s["lr"] * s["decay"]) * s["w"] - (s["lr"] * s["scale"]) * o
    return {"w": w, "momentum": m, "w_bf16": w.to(torch.bfloat16)}


# ---- inputs -----------------------------------------------------------------------------------------------------------

def _rand(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std)


def _activation(gen, rows, cols):
    x = _rand(gen, rows, cols)
    x[:, torch.randperm(cols, generator=gen, device="cuda")[:16]] *= 50.0
    return x


def _weight_gradient(gen, rows, cols):
    """What the products of 24 strong tokens and the noise of all others leave."""
    return _rand(gen, rows, cols, std=1e-4).addmm_(_rand(gen, rows, 24, std=3e-4), _activation(gen, cols, 24).t(), alpha=0.3)


def _prepare_ce(gen, case):
    T, D, V = case["tokens"], case["dim"], case["vocab"]
    s = {"h": _activation(gen, T, D).to(torch.bfloat16), "w": _rand(gen, V, D, std=0.02).to(torch.bfloat16),
         "logit_scale": case["logit_scale"], "z_loss": case["z_loss"]}
    targets = torch.randint(0, V, (T,), generator=gen, device="cuda")
    s["targets"] = torch.where(torch.rand(T, generator=gen, device="cuda") < case["ignored"], IGNORED, targets)
    if case["kind"] == "ce_fwd":
        s["out"] = {k: torch.empty(T, dtype=torch.float32, device="cuda") for k in ("loss", "lse")}
        return s
    w = s["w"].float().t()
    s["lse"] = torch.cat([torch.logsumexp((s["h"][i:i + 4096].float() @ w) * s["logit_scale"], 1) for i in range(0, T, 4096)])
    s["d_loss"] = (1.0 / (s["targets"] >= 0).sum().clamp(min=1).float()).expand(T)       # of the mean over the tokens that count
    s["out"] = {"d_h": torch.empty_like(s["h"]), "d_w": torch.empty_like(s["w"])}
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    if kind.startswith("ce"):
        return {"kind": kind} | _prepare_ce(gen, case)
    rows, cols = case["rows"], case["cols"]
    s = {"kind": kind, "g": _weight_gradient(gen, rows, cols).to(torch.float32 if case["f32"] else torch.bfloat16)}
    if kind == "orth":
        return s | {"out": torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")}
    w = _rand(gen, rows, cols, std=0.02)
    # a rate as it is with other optimizers, whose step this scale has: 0.2 of the rate for each element
    return s | {"w": w, "momentum": _weight_gradient(gen, rows, cols).mul_(4.0), "lr": 1e-4, "scale": 0.2 * math.sqrt(max(rows, cols)),
                "nesterov": case["nesterov"], "decay": case["decay"],
                "out": {"w_out": torch.empty_like(w), "momentum_out": torch.empty_like(w), "w_bf16": torch.empty_like(w, dtype=torch.bfloat16)}}


# ---- one pass ---------------------------------------------------------------------------------------------------------

def _own(s):
    from paper_2604_02525_amd import binding as ah
    kind = s["kind"]
    if kind == "ce_fwd":
        return ah.adahop_linear_ce(s["h"], s["w"], s["targets"], logit_scale=s["logit_scale"], z_loss=s["z_loss"], **s["out"])
    if kind == "ce_bwd":
        return ah.adahop_linear_ce_backward(s["h"], s["w"], s["targets"], s["lse"], s["d_loss"], logit_scale=s["logit_scale"], z_loss=s["z_loss"], **s["out"])
    if kind == "orth":
        return {"out": ah.adahop_orthogonalize(s["g"], out=s["out"], steps=STEPS, coefficients=COEFFICIENTS, eps=EPS)}
    return ah.adahop_muon_update(s["w"], s["g"], s["momentum"], s["lr"], mu=MU, weight_decay=s["decay"], nesterov=s["nesterov"], scale=s["scale"], steps=STEPS,
                                 coefficients=COEFFICIENTS, eps=EPS, **s["out"])


def run(state):
    if own:
        return _own(state)
    return {"ce_fwd": _ce_fwd_out, "ce_bwd": _ce_bwd_out, "orth": _orth_out, "muon": _muon_out}[state["kind"]](state)


def work(case):
    if case["kind"].startswith("ce"):
        T, D, V = case["tokens"], case["dim"], case["vocab"]
        once = 2 * (T * D + V * D) + 8 * T
        if case["kind"] == "ce_fwd":
            return {"bytes": once + 8 * T, "flops": 2 * T * D * V}
        return {"bytes": 2 * once, "flops": 6 * T * D * V}       # the logits again, then both gradients
    m, n = sorted((case["rows"], case["cols"]))
    flops = STEPS * (m * m * n + m * m * m + 2 * m * m * n)      # half of each of the two symmetric products
    g = 4 if case["f32"] else 2
    return {"bytes": m * n * (g + 2 if case["kind"] == "orth" else g + 4 + 4 + 4 + 4 + 2), "flops": flops}


# ---- in 64 bits -------------------------------------------------------------------------------------------------------

def _exact_step(u):
    """The polynomial of the method on the singular directions, products in 64 bits."""
    a, b, c = COEFFICIENTS
    x = u / (torch.linalg.vector_norm(u) + EPS)
    right = x.shape[1] <= x.shape[0]
    for _ in range(STEPS):
        gram = x.mT @ x if right else x @ x.mT
        p = torch.addmm(gram, gram, gram, beta=b, alpha=c)
        p.diagonal().add_(a)
        x = x @ p if right else p @ x
    return x


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "orth":
        return {"out": _exact_step(s["g"].double())}
    if kind == "muon":
        g = s["g"].double()
        m = s["momentum"].double().mul_(MU).add_(g)
        o = _exact_step(torch.add(g, m, alpha=MU) if s["nesterov"] else m)
        w = s["w"].double().mul_(1.0 - s["lr"] * s["decay"]).sub_(o, alpha=s["lr"] * s["scale"])
        return {"w": w, "momentum": m, "w_bf16": w}
    T = case["tokens"]
    h, w, targets, rows = s["h"].double(), s["w"].double(), s["targets"], torch.arange(T, device="cuda")
    z = torch.matmul(h, w.mT).mul_(s["logit_scale"])
    counts, safe = targets.ge(0), targets.clamp_min(0)
    if kind == "ce_fwd":
        lse = torch.logsumexp(z, 1)
        return {"loss": (lse - z[rows, safe] + s["z_loss"] * lse.square()).masked_fill(~counts, 0.0), "lse": lse}
    lse = s["lse"].double()
    p = z.sub_(lse[:, None]).exp_().mul_(1.0 + 2.0 * s["z_loss"] * lse[:, None])
    p[rows, safe] -= 1.0
    p.mul_((s["d_loss"].double() * s["logit_scale"]).masked_fill(~counts, 0.0)[:, None])
    return {"d_h": p @ w, "d_w": p.mT @ h}
