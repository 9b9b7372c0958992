"""Gradients of the label loss that were computed in the forward call, under an upstream gradient that is not 1."""
import pytest
import torch

from paper_2608_03796_b200.autograd import label_loss

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("T,H,V", [(1, 64, 33), (40, 128, 1001), (300, 264, 2001)])
@pytest.mark.parametrize("factor", [1.0, 1 / 3, -0.7, 1e-3, 0.0])
def test_one_more_rounding(T, H, V, factor):
    """The finished gradient times the factor in fp32, rounded once: that, bit for bit."""
    g = torch.Generator(device="cuda").manual_seed(T)
    h = torch.randn(T, H, generator=g, device="cuda").to(BF16)
    w = (torch.randn(V, H, generator=g, device="cuda") / H ** 0.5).to(BF16)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")

    def grads(up):
        a, b = h.clone().requires_grad_(), w.clone().requires_grad_()
        loss = label_loss(a, b, y, single_pass=True)
        loss.backward(torch.tensor(up, device="cuda"), retain_graph=True)
        first = a.grad.clone(), b.grad.clone()
        a.grad = b.grad = None
        loss.backward(torch.tensor(up, device="cuda"))                      # the finished ones are still whole
        assert torch.equal(a.grad, first[0]) and torch.equal(b.grad, first[1])
        return first
    whole = grads(1.0)
    for got, one in zip(grads(factor), whole):
        assert got.dtype == BF16 and torch.equal(got, (one.float() * torch.tensor(factor, device="cuda")).to(BF16))


def test_one_gradient_alone():
    h, w, y = torch.randn(50, 64, device="cuda").to(BF16), torch.randn(70, 64, device="cuda").to(BF16), torch.arange(50, device="cuda")
    a = h.clone().requires_grad_()
    label_loss(a, w, y, single_pass=True).backward()
    b = h.clone().requires_grad_()
    (label_loss(b, w, y, single_pass=True) / 3).backward()
    third = torch.tensor(1.0, device="cuda") / 3
    assert torch.equal(b.grad, (a.grad.float() * third).to(BF16))


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("rows", [0, 1, 33, 5000])
def test_the_product_alone(dtype, rows):
    """Values of any kind; a factor that is not finite; the last word; an output beside its neighbours."""
    from paper_2608_03796_b200.labels import rescaled
    t = torch.randn(rows, 24, device="cuda").to(dtype)
    if rows:
        t[0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 0.0])
    for factor in (1 / 3, -0.0, float("inf")):
        f = torch.tensor(factor, device="cuda")
        got, want = rescaled(t, f), (t.float() * f).to(dtype)
        assert got.data_ptr() != t.data_ptr() or not rows
        assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0)) and torch.equal(got.isnan(), want.isnan())
    for bad in (lambda: rescaled(t.cpu(), f), lambda: rescaled(t, f.double()), lambda: rescaled(t, f.cpu())):
        with pytest.raises(TypeError):
            bad()
