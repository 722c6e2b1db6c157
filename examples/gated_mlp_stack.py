"""A stack of gated MLP blocks trained with MXFP4 products (forward and input gradients), its activations kept in 8 bits.

    python examples/gated_mlp_stack.py --tokens 4096 --hidden 2048 --ffn 5632 --blocks 4 --steps 10
    python examples/gated_mlp_stack.py --tokens 4096 --hidden 2048 --ffn 5632 --blocks 4 --steps 10 --vocab 32000

Each block is  h -> [g | u] = h W_gu^T -> a = silu(g) u -> y = a W_down^T,  and between two blocks

    s' = residual_scale s + gate * w_post * norm(y),   h' = w_pre * norm(s').

The products of a block run as MXFP4 (adahop_gemm).  What lies between them runs in one pass over the memory each, and leaves behind what the
backward pass takes: norm(s') and norm(y) in 8 bits, g and u in 8 bits, two numbers per row.  Of all activations only these are kept, 33/32 bytes an
element; a is formed again from g and u by the backward pass, and the weight gradients are computed from the 8-bit
rows, in bf16: nothing is rounded to 4 bits on the way into the float32 gradient. Where speed counts for more, adahop_ckpt8_unpack and an
MXFP4 product take less than half of the time for large layers.  The one checkpoint of norm(s') serves the gradient of W_gu (times w_pre, feature by feature) and the norm's own backward pass.

With --vocab the stack ends in the loss of one word per token (adahop_linear_ce: h times bf16 output weights, the logits never in memory), and the matrices of the blocks are updated by
their orthogonalised momentum (adahop_muon_update), which leaves the next step's bf16 weights behind; the vectors and the output weights take the plain step.
"""
import argparse
import os
import sys
import time

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2604_02525_amd import binding as ah  # noqa: E402


class GatedMlpStack:
    """hidden and ffn are multiples of 32 (of iht_block if that is larger).  Weights are bfloat16 with float32 masters; `grads` holds
    their float32 gradients, which backward() adds to once accumulate is set."""

    def __init__(self, hidden, ffn, blocks, iht_block=32, residual_scale=1.0, seed=0, device="cuda", vocab=0):
        self.hidden, self.ffn, self.blocks, self.iht_block, self.residual_scale = hidden, ffn, blocks, iht_block, residual_scale
        draw = torch.Generator(device=device).manual_seed(seed)
        self.masters = {}
        for b in range(blocks):
            self.masters[f"gu{b}"] = torch.randn(2 * ffn, hidden, generator=draw, device=device) * hidden ** -0.5
            self.masters[f"down{b}"] = torch.randn(hidden, ffn, generator=draw, device=device) * ffn ** -0.5
            self.masters[f"pre{b}"] = torch.ones(hidden, device=device)
            self.masters[f"post{b}"] = torch.ones(hidden, device=device)
            self.masters[f"gate{b}"] = torch.full((hidden,), 0.5, device=device)
        self.masters[f"pre{blocks}"] = torch.ones(hidden, device=device)
        if vocab:
            self.masters["out"] = torch.randn(vocab, hidden, generator=draw, device=device) * hidden ** -0.5
        self.momentum = {}
        self.grads = {k: torch.zeros_like(w) for k, w in self.masters.items()}  # (the output weights stay as they are in steps without words)
        self.round_weights()

    def round_weights(self):
        self.w = {k: m.to(torch.bfloat16) if m.dim() == 2 else m for k, m in self.masters.items()}

    def product(self, a, b, b_k_contig):
        """a [tokens, K] times b: [N, K] (b_k_contig) or [K, N]; bfloat16."""
        return ah.adahop_gemm(ah.Operand(a, True), ah.Operand(b, b_k_contig), ah.ADAHOP_IHT, self.iht_block, c_bf16=True)["C"]

    def forward(self, x):
        """(h after the last block, what backward takes)"""
        w, joins, acts = self.w, [], []
        joins.append(ah.adahop_block_norm(x, w_pre=w["pre0"], keep="ckpt8"))
        for b in range(self.blocks):
            gu = self.product(joins[b].pop("h"), w[f"gu{b}"], True)
            act = ah.adahop_swiglu(gu[:, :self.ffn], gu[:, self.ffn:], keep8=True)
            y = self.product(act.pop("a"), w[f"down{b}"], True)
            acts.append(act)
            joins.append(ah.adahop_block_norm(joins[b].pop("s"), y, w_post=w[f"post{b}"], w_pre=w[f"pre{b + 1}"], gate=w[f"gate{b}"],
                                              residual_scale=self.residual_scale, keep="ckpt8"))
        joins[-1].pop("s")
        return joins[-1].pop("h"), (joins, acts)

    def join_backward(self, b, d_s, d_h, join, accumulate):
        names = {"d_w_pre": f"pre{b}"}
        given = {}
        if b:
            names.update(d_w_post=f"post{b - 1}", d_gate=f"gate{b - 1}")
            given = dict(w_post=self.w[f"post{b - 1}"], gate=self.w[f"gate{b - 1}"], residual_scale=self.residual_scale)
        into = {k: torch.empty_like(self.grads[n]) if accumulate else self.grads[n] for k, n in names.items()}
        out = ah.adahop_block_norm_backward(d_s, d_h, join["ckpt_s"], join["ckpt_y"], join["rstd_pre"], join["rstd_post"], w_pre=self.w[f"pre{b}"],
                                            **given, **into)
        if accumulate:
            for k, n in names.items():
                self.grads[n] += into[k]
        return out["d_x"], out["d_y"]

    def weight_gradient(self, name, d_out, x8, col_scale, accumulate):
        ah.adahop_ckpt8_wgrad(d_out, x8, col_scale=col_scale, add=self.grads[name] if accumulate else None, Cout=self.grads[name])

    def backward(self, d_h, kept, accumulate=False):
        """Fills (accumulate: adds to) grads; returns the gradient of x."""
        joins, acts = kept
        d_s = None
        for b in reversed(range(self.blocks)):
            d_s, d_y = self.join_backward(b + 1, d_s, d_h, joins[b + 1], accumulate)
            g8, u8 = acts[b]["ckpt_g"], acts[b]["ckpt_u"]
            d_a = self.product(d_y, self.w[f"down{b}"], False)
            d_gu = torch.empty(d_a.shape[0], 2 * self.ffn, dtype=torch.bfloat16, device=d_a.device)
            a8 = ah.adahop_swiglu_backward(g8, u8, d_a, d_g=d_gu[:, :self.ffn], d_u=d_gu[:, self.ffn:],
                                           a=ah.adahop_ckpt8_empty(*d_a.shape, device=d_a.device))["a"]
            self.weight_gradient(f"down{b}", d_y, a8, None, accumulate)
            self.weight_gradient(f"gu{b}", d_gu, joins[b]["ckpt_s"], self.w[f"pre{b}"], accumulate)
            d_h = self.product(d_gu, self.w[f"gu{b}"], False)
        d_x, _ = self.join_backward(0, d_s, d_h, joins[0], accumulate)
        return d_x

    def update(self, rate):
        """Each tensor a step of `rate` times its own magnitude against its gradient."""
        for k, m in self.masters.items():
            g = self.grads[k]
            m -= g * (rate * m.norm() / g.norm().clamp(min=1e-30))
        self.round_weights()

    def step(self, x, target, rate):
        """One step towards h = target; returns half the mean squared distance before it (a tensor)."""
        h, kept = self.forward(x)
        off = h.float() - target
        self.backward((off / off.numel()).to(torch.bfloat16), kept)
        self.update(rate)
        return off.square().mean() / 2

    def words_loss_and_gradients(self, x, words):
        """Mean loss of predicting `words` (int64 per token, negative: none) from h, a tensor; fills grads."""
        h, kept = self.forward(x)
        f = ah.adahop_linear_ce(h, self.w["out"], words)
        each = 1.0 / (words >= 0).sum().clamp(min=1).float()
        d_h = ah.adahop_linear_ce_backward(h, self.w["out"], words, f["lse"], each.expand(len(words)), d_w=self.grads["out"])["d_h"]
        self.backward(d_h, kept)
        return f["loss"].sum() * each

    def orthogonal_update(self, rate, scale=0.02):
        """The blocks' matrices a step of `scale * rate` per element along their orthogonalised momentum, all else as in update()."""
        for k, m in self.masters.items():
            if m.dim() == 2 and k != "out":
                momentum = self.momentum.setdefault(k, torch.zeros_like(m))
                ah.adahop_muon_update(m, self.grads[k], momentum, rate, scale=scale * max(m.shape) ** 0.5, w_bf16=self.w[k])
            else:
                m -= self.grads[k] * (rate * m.norm() / self.grads[k].norm().clamp(min=1e-30))
                self.w[k] = m.to(torch.bfloat16) if m.dim() == 2 else m

    def words_step(self, x, words, rate):
        loss = self.words_loss_and_gradients(x, words)
        self.orthogonal_update(rate)
        return loss


def kept_bytes(kept):
    """Bytes of all that forward() leaves for the backward pass."""
    total = 0
    for part in [*kept[0], *kept[1]]:
        for v in part.values():
            total += sum(t.numel() * t.element_size() for t in (v if isinstance(v, tuple) else (v,)) if t is not None)
    return total


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("tokens", 4096), ("hidden", 2048), ("ffn", 5632), ("blocks", 4), ("steps", 10), ("iht-block", 32)):
        p.add_argument("--" + name, type=int, default=default)
    p.add_argument("--rate", type=float, default=0.02)
    p.add_argument("--vocab", type=int, default=0)
    a = p.parse_args()
    ah.adahop_prepare_device()
    net = GatedMlpStack(a.hidden, a.ffn, a.blocks, a.iht_block, vocab=a.vocab)
    draw = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(a.tokens, a.hidden, generator=draw, device="cuda").to(torch.bfloat16)
    target = torch.randint(0, a.vocab, (a.tokens,), generator=draw, device="cuda") if a.vocab else x.float().roll(1, 1)
    kept = net.forward(x)[1]
    elements = a.tokens * a.blocks * (2 * a.hidden + 2 * a.ffn) + a.tokens * a.hidden
    print(f"kept for the backward pass: {kept_bytes(kept) / 2**20:.1f} MiB ({kept_bytes(kept) / elements:.3f} bytes an element)", flush=True)
    del kept
    for i in range(a.steps):
        torch.cuda.synchronize()
        t = time.perf_counter()
        loss = (net.words_step if a.vocab else net.step)(x, target, a.rate)
        torch.cuda.synchronize()
        print(f"step {i}: loss {loss.item():.5f}, {(time.perf_counter() - t) * 1e3:.2f} ms", flush=True)


if __name__ == "__main__":
    main()
