"""The holders' buffers for gradients of weights. No GPU needed."""
import pytest
import torch

from paper_2608_03796_b200 import body

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("made", [lambda: body.LayerNorm(4, 64, device="cpu"), lambda: body.BlockNorm(4, 64, device="cpu")])
def test_gradient_buffers_of_both_weight_types_stay(made):
    """A buffer that a kernel of another stream may still write is not given up because a weight of another type came."""
    op, w = made(), torch.ones(64)
    a = op._grad("weight", w.to(BF16))
    b = op._grad("weight", w)
    assert a.dtype == BF16 and b.dtype == F32
    assert op._grad("weight", w.to(BF16)) is a and op._grad("weight", w) is b
