"""The mean of the layer norm's fp32 rows: of equal values it is the value, of values far from zero their mean to the last bit or
so, however the sum was rounded on the way.

The first sum's mean m is off by the rounding of the sum. The values less m are exact where they are near it (within a factor
of two of one another, as fp32 numbers), and their own mean is what m lacks, off by a share of itself: the corrected mean is
rounded once more and nothing else of that size remains. Tolerance of the mean: that rounding and C = 64 units of the values' spread
around it."""
import pytest
import torch

from paper_2608_03796_b200 import body

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
UNIT, C = 2.0 ** -24, 64
# a warp's rows (whole words, and not), a block's (whole trips, part-filled ones, element by element), wider ones
WIDTHS = [1, 7, 200, 257, 512, 1000, 2880, 4096, 4095, 8192, 8200, 9001, 40000, 100001]


@pytest.mark.parametrize("H", WIDTHS)
@pytest.mark.parametrize("x_type,type", [(F32, F32), (F32, BF16), (BF16, BF16), (F16, F16)])
def test_equal_values(H, x_type, type):
    """xh = 0, y = bias, exactly; dx of such a row is rho (g - mean g) and the row adds nothing to dweight."""
    T = 24
    g = torch.Generator(device="cuda").manual_seed(H)
    values = 405.55185 * (2 * torch.rand(T, generator=g, device="cuda") - 1)
    x = values.to(x_type)[:, None].expand(T, H).contiguous()
    w, b = torch.randn(H, generator=g, device="cuda"), torch.randn(H, generator=g, device="cuda")
    op = body.LayerNorm(T, H, dtype=type, x_dtype=x_type, eps=1e-5)
    y = op.forward(x, w, b)
    assert torch.equal(op.stats[0], x[:, 0].float())
    assert torch.equal(y, b.to(type).expand(T, H))
    d = op.backward(torch.randn(T, H, generator=g, device="cuda").to(type))
    assert not d.weight.any()


@pytest.mark.parametrize("H", [200, 257, 1000, 2880, 4096, 4095, 9001])
def test_values_far_from_zero(H):
    T = 40
    g = torch.Generator(device="cuda").manual_seed(H)
    x = 1000 + 0.01 * torch.randn(T, H, generator=g, device="cuda")
    op = body.LayerNorm(T, H, dtype=F32, eps=1e-9)
    y = op.forward(x)
    X = x.double()
    mean, spread = X.mean(1), X.std(1, unbiased=False)
    off = 1.001 * 2.0 ** -15 + C * UNIT * spread                            # (half a unit of [512, 1024), where the means lie)
    assert float(((op.stats[0].double() - mean).abs() - off).max()) <= 0
    rho = ((X - mean[:, None]).square().mean(1) + 1e-9) ** -0.5
    xh = (X - mean[:, None]) * rho[:, None]
    bound = rho[:, None] * off[:, None] + C * UNIT * (1 + xh.abs()) + (rho * off)[:, None] ** 2 * xh.abs()
    assert float(((y.double() - xh).abs() - bound - xh.abs() * UNIT).max()) <= 0
