"""The backward passes are differentiated once. Under create_graph a gradient that depends on them further says so when it
is differentiated, whether or not the upstream gradient needed a graph; before, the terms were missing without a word."""
import pytest
import torch

from paper_2608_03796_b200 import autograd as A

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _randn(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(BF16)


def _functions():
    T, H, V = 40, 64, 128
    x, w = _randn(1, T, H).requires_grad_(True), _randn(2, V, H).requires_grad_(True)
    z, one = _randn(3, T, 2 * H).requires_grad_(True), torch.ones(H, dtype=BF16, device="cuda")
    idx = torch.arange(4, dtype=torch.int32, device="cuda").repeat(T, 1)
    val = torch.zeros(T, 4, device="cuda")
    return {
        "act8_linear": (lambda: A.act8_linear(x, w), (x, w)),
        "gated_act": (lambda: A.gated_act(z), (z,)),
        "block_norm": (lambda: sum(A.block_norm(x, 2 * x, one, one, act8="int8")), (x,)),
        "fused_chunked_kl": (lambda: A.fused_chunked_kl(x, w, idx, val, chunk=16), (x, w)),
        "feature_loss": (lambda: A.feature_loss(x, x.detach() + 1), (x,)),
    }


@pytest.mark.parametrize("name", ["act8_linear", "gated_act", "block_norm", "fused_chunked_kl", "feature_loss"])
@pytest.mark.parametrize("upstream", ["constant", "graph"])
def test_second_derivatives_are_refused(name, upstream):
    f, leaves = _functions()[name]
    y = f()
    # first derivatives under create_graph are what they are without
    plain = torch.autograd.grad((y if upstream == "constant" else y * y).sum(), leaves, retain_graph=True)
    y = f()
    grads = torch.autograd.grad((y if upstream == "constant" else y * y).sum(), leaves, create_graph=True)
    for g, p in zip(grads, plain):
        assert torch.equal(g, p)
    penalty = sum((g.float() ** 2).sum() for g in grads) + sum((t.float() ** 2).sum() for t in leaves)
    with pytest.raises(RuntimeError, match=f"{name}.*second"):
        penalty.backward()
