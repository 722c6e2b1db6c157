"""The example's plain step on a stack that has output weights: what no gradient has been formed of stays as it is."""
import pytest

import test_gpu_gated_mlp_example as stack

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
example = stack.example


def test_a_step_without_words_leaves_the_output_weights(example):
    room = [torch.full((1001, 128), float("nan"), device="cuda") for _ in range(8)]     # what memory of that size held before
    del room
    net = example.GatedMlpStack(128, 384, 1, vocab=1001)
    before = net.masters["out"].clone()
    x = torch.randn(256, 128, device="cuda").to(torch.bfloat16)
    net.step(x, x.float().roll(1, 1), 0.02)
    assert torch.equal(net.masters["out"], before) and torch.equal(net.w["out"], before.to(torch.bfloat16))
