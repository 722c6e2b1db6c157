"""The loss over a vocabulary where a batch has nothing to learn from: what one d_loss for all tokens holds takes no part without a token that has a target, as that of a token without one does
not.  (A mean over no tokens has the gradient 1 / 0.)"""
import pytest

import test_gpu_linear_ce as many

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ah = many.ah


# few tokens; tiles of both sizes; slices that a second kernel joins
@pytest.mark.parametrize("T,D,V", [(1, 40, 50), (8, 64, 200), (50, 72, 200), (3000, 256, 300)])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_no_target_and_one_gradient_that_is_not_finite(ah, T, D, V, value):
    many.say("no target", T, D, V, value)
    h, w = torch.randn(T, D, device="cuda").to(torch.bfloat16), torch.randn(V, D, device="cuda").to(torch.bfloat16)
    targets, lse = torch.full((T,), -100, device="cuda"), torch.zeros(T, device="cuda")
    one = torch.full((1,), value, device="cuda").expand(T)
    out = ah.adahop_linear_ce_backward(h, w, targets, lse, one)
    assert not out["d_h"].any() and not out["d_w"].any()
    add = torch.randn(V, D, device="cuda")
    out = ah.adahop_linear_ce_backward(h, w, targets, lse, one, add=add)
    assert torch.equal(out["d_w"], add)
    each = torch.full((T,), value, device="cuda")
    assert torch.equal(ah.adahop_linear_ce_backward(h, w, targets, lse, each, add=add)["d_w"], add)
    targets[T // 2] = 3                     # one token that has one: its own gradients are not finite, nobody else's
    out = ah.adahop_linear_ce_backward(h, w, targets, lse, one)
    assert not out["d_h"][T // 2].isfinite().any() and not out["d_w"].isfinite().any()
    out["d_h"][T // 2] = 0
    assert not out["d_h"].any()
