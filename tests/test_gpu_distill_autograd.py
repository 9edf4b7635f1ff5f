"""The gradient in place of the logits, beside autograd."""
import pytest
import torch

import paper_2409_16560_b200 as dsbd
import rows_util as ru

pytestmark = pytest.mark.gpu


def problem():
    value, index, rest, _ = dsbd.top_logits(ru.rows_of(4, 300, torch.float32, seed=1), 10)
    h = torch.randn(4, 16, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    W = torch.randn(16, 300, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).requires_grad_()
    return h, W, value, index, rest


def test_in_place_behind_a_product():
    """A product does not need its result again: the gradients are those of the call into a tensor of its own."""
    h, W, value, index, rest = problem()
    logits = h @ W
    _, grad, _ = dsbd.distill(logits, value, index, rest=rest)
    want, = torch.autograd.grad(logits, W, grad)
    logits = h @ W
    _, grad, _ = dsbd.distill(logits, value, index, rest=rest, grad=logits)
    assert grad is logits
    got, = torch.autograd.grad(logits, W, grad.detach())
    assert torch.equal(got, want)


@pytest.mark.parametrize("view", [False, True])
def test_in_place_where_the_logits_are_needed_again(view):
    """A soft cap's backward reads its result: overwritten logits are refused there."""
    h, W, value, index, rest = problem()
    logits = 30 * torch.tanh(h @ W / 30)
    capped = torch.tanh(h @ W)
    _, grad, _ = dsbd.distill(capped, value, index, rest=rest, grad=capped.detach() if view else capped)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        capped.backward(grad.detach().clone())
    _, grad, _ = dsbd.distill(logits, value, index, rest=rest, grad=logits)
    logits.backward(grad.detach())                             # the product with 30 keeps tanh's result, not its own
    assert bool(W.grad.isfinite().all())
