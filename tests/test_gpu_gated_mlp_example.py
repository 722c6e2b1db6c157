"""The example that trains gated MLP blocks: its gradients against those of the same network in 64 bits, and that it learns.

Bound of the gradients, with products in fp32 rounded to bf16 in place of the MXFP4 ones: any term of a gradient holds at most three factors
that were kept in 8 bits (the norms of both sides, and g or u), each off by at most 1/16 of itself, independently of the others: sqrt(3) / 16 of its Frobenius norm
for one block.  Further blocks add their own share: sqrt(3 blocks) / 16.  bf16's half steps (2^-8, some twenty to a block) stay below 2^-8 sqrt(20 blocks)."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_mlp_stack.py")


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("gated_mlp_stack", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(net, x, d_h):
    """Gradients of <h, d_h> in 64 bits on the CPU."""
    w = {k: v.double().cpu().requires_grad_() for k, v in net.w.items()}
    x = x.double().cpu().requires_grad_()

    def norm(v):
        return v / (v.square().mean(1, keepdim=True) + 1e-6).sqrt()
    s, h = x, norm(x) * w["pre0"]
    for b in range(net.blocks):
        g, u = (h @ w[f"gu{b}"].T).split(net.ffn, dim=1)
        y = (torch.nn.functional.silu(g) * u) @ w[f"down{b}"].T
        s = net.residual_scale * s + w[f"gate{b}"] * w[f"post{b}"] * norm(y)
        h = norm(s) * w[f"pre{b + 1}"]
    (h * d_h.double().cpu()).sum().backward()
    return h.detach(), x.grad, {k: v.grad for k, v in w.items()}


def relative(got, want):
    return ((got.double().cpu() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("tokens,hidden,ffn,blocks", [(96, 64, 160, 1), (200, 128, 320, 2), (1, 64, 96, 1)])
def test_gradients_of_the_stack(example, tokens, hidden, ffn, blocks):
    print("[case]", tokens, hidden, ffn, blocks, flush=True)

    class Plain(example.GatedMlpStack):
        def product(self, a, b, b_k_contig):
            return (a.float() @ (b.float().T if b_k_contig else b.float()).contiguous()).to(torch.bfloat16)
    net = Plain(hidden, ffn, blocks, residual_scale=0.75)
    draw = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(tokens, hidden, generator=draw, device="cuda").to(torch.bfloat16)
    d_h = torch.randn(tokens, hidden, generator=draw, device="cuda").to(torch.bfloat16)
    h, kept = net.forward(x)
    d_x = net.backward(d_h, kept)
    want_h, want_x, want = reference(net, x, d_h)
    bound = (3 * blocks) ** 0.5 / 16 + (20 * blocks) ** 0.5 / 256
    assert relative(h, want_h) < (20 * blocks) ** 0.5 / 256
    assert relative(d_x, want_x) < bound
    for k, g in net.grads.items():
        assert relative(g, want[k]) < bound, k
    once = {k: g.clone() for k, g in net.grads.items()}
    net.backward(d_h, kept, accumulate=True) # a second micro-batch, here the same one
    for k, g in net.grads.items():
        assert torch.allclose(g, 2 * once[k], rtol=1e-5, atol=1e-5 * once[k].abs().max().item()), k


def test_the_stack_learns_with_mxfp4_products(example):
    """Twenty steps of 2 % against the gradient take more than a tenth off the loss."""
    net = example.GatedMlpStack(128, 384, 2)
    draw = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(512, 128, generator=draw, device="cuda").to(torch.bfloat16)
    target = x.float().roll(1, 1)
    losses = [net.step(x, target, 0.02).item() for _ in range(20)]
    print("losses", losses, flush=True)
    assert losses[-1] < 0.9 * losses[0]


def test_what_the_stack_keeps(example):
    """33/32 bytes an element of norm(s), norm(y), g and u, two numbers a row beside them, and nothing else."""
    net = example.GatedMlpStack(256, 512, 3)
    x = torch.randn(64, 256, device="cuda").to(torch.bfloat16)
    kept = net.forward(x)[1]
    elements = 64 * (3 * (2 * 256 + 2 * 512) + 256)
    assert example.kept_bytes(kept) == elements * 33 // 32 + 64 * 4 * (2 * 3 + 1)
