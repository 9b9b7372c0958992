"""The guard of backward passes that cannot be differentiated, on a Function of the host's."""
import pytest
import torch

from paper_2608_03796_b200 import autograd as A


class _Square(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y):
        ctx.save_for_backward(x)
        return x * x

    @staticmethod
    @A._first_derivative_only("square")
    def backward(ctx, g):
        (x,) = ctx.saved_tensors
        return 2 * x * g, None


@pytest.mark.parametrize("upstream", ["constant", "graph"])
def test_a_gradient_of_a_gradient_raises(upstream):
    x = torch.tensor([1.0, 2.0], requires_grad=True)
    y = _Square.apply(x, None)
    loss = y.sum() if upstream == "constant" else (y * y).sum()
    (g,) = torch.autograd.grad(loss, x, create_graph=True)
    assert torch.equal(g.detach(), 2 * x.detach() if upstream == "constant" else 4 * x.detach() ** 3)
    with pytest.raises(RuntimeError, match="square.*second"):
        ((g ** 2).sum() + (x ** 2).sum()).backward()
    loss = _Square.apply(x, None).sum()
    x.grad = None
    loss.backward()                                                         # the first derivative is as it was
    assert torch.equal(x.grad, 2 * x.detach()) and not x.grad.requires_grad


@pytest.mark.parametrize("function", [A._FusedChunkedKL, A._FeatureLoss, A._Act8Linear, A._GatedAct, A._BlockNorm])
def test_every_backward_pass_has_the_guard(function):
    assert hasattr(function.backward, "__wrapped__")
