"""The example that trains gated MLP blocks, ending in the loss over a vocabulary: its gradients against those of the same network in 64 bits, and that its steps run.

Bound of the gradients: as for the stack alone (sqrt(3 blocks) / 16 of a gradient's norm for what is kept in 8 bits, sqrt(20 blocks) / 256 for the roundings to bf16), and of the gradient
that enters it, two roundings to bf16 more."""
import pytest

import test_gpu_gated_mlp_example as stack

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
example = stack.example


def reference(net, x, words):
    """Mean loss and gradients in 64 bits on the CPU."""
    w = {k: v.double().cpu().requires_grad_() for k, v in net.w.items()}

    def norm(v):
        return v / (v.square().mean(1, keepdim=True) + 1e-6).sqrt()
    s = x.double().cpu()
    h = norm(s) * w["pre0"]
    for b in range(net.blocks):
        g, u = (h @ w[f"gu{b}"].T).split(net.ffn, dim=1)
        y = (torch.nn.functional.silu(g) * u) @ w[f"down{b}"].T
        s = net.residual_scale * s + w[f"gate{b}"] * w[f"post{b}"] * norm(y)
        h = norm(s) * w[f"pre{b + 1}"]
    loss = torch.nn.functional.cross_entropy(h @ w["out"].T, words.cpu(), ignore_index=-100)
    loss.backward()
    return loss.item(), {k: v.grad for k, v in w.items()}


def inputs(net, tokens, vocab, seed=5):
    draw = torch.Generator(device="cuda").manual_seed(seed)
    words = torch.randint(0, vocab, (tokens,), generator=draw, device="cuda")
    words[1::7] = -100
    return torch.randn(tokens, net.hidden, generator=draw, device="cuda").to(torch.bfloat16), words


@pytest.mark.parametrize("tokens,hidden,ffn,blocks,vocab", [(96, 64, 160, 1, 300), (200, 128, 320, 2, 1001)])
def test_gradients_of_the_words_loss(example, tokens, hidden, ffn, blocks, vocab):
    print("[case]", tokens, hidden, ffn, blocks, vocab, flush=True)

    class Plain(example.GatedMlpStack):
        def product(self, a, b, b_k_contig):
            return (a.float() @ (b.float().T if b_k_contig else b.float()).contiguous()).to(torch.bfloat16)
    net = Plain(hidden, ffn, blocks, residual_scale=0.75, vocab=vocab)
    x, words = inputs(net, tokens, vocab)
    loss = net.words_loss_and_gradients(x, words).item()
    want_loss, want = reference(net, x, words)
    bound = (3 * blocks) ** 0.5 / 16 + (20 * blocks + 2) ** 0.5 / 256
    assert abs(loss - want_loss) < (20 * blocks) ** 0.5 / 256 * want_loss
    for k, g in net.grads.items():
        assert stack.relative(g, want[k]) < bound, k


def test_steps_run_and_move_the_weights(example):
    """Masters, momentum and the bf16 weights of the next products go together."""
    net = example.GatedMlpStack(128, 384, 2, vocab=1001)
    x, words = inputs(net, 512, 1001)
    before = {k: m.clone() for k, m in net.masters.items()}
    for _ in range(3):
        loss = net.words_step(x, words, 0.02)
    assert torch.isfinite(loss)
    for k, m in net.masters.items():
        assert torch.isfinite(m).all() and not torch.equal(m, before[k]), k
        assert torch.equal(net.w[k], m.to(torch.bfloat16) if m.dim() == 2 else m), k
    assert set(net.momentum) == {"gu0", "down0", "gu1", "down1"}
