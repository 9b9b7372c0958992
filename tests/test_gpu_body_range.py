"""The ends of a record's range, exactly.

Top: a group whose largest value would, rounded to nearest, read back as 2^128 takes the code below: 63 * 2^122 (int8) and
240 * 2^120 (e4m3). Bottom: the exponent stops at -126, so a group's step is then fixed whatever its largest value:
2^-126 (int8) and 2^-135 (the least e4m3 code); bf16 ends at 2^-133, so the least e4m3 values are rounded where they are read
as bf16: by load and by the weight gradient on the tensor cores. The element-wise weight gradient reads them in fp32, exactly.
"""
import numpy as np
import pytest
import torch

from oracle import body_oracle as O
from paper_2608_03796_b200 import body

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
TOP = {"int8": 63 * 2.0 ** 122, "e4m3": 240 * 2.0 ** 120}


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H", [64, 63])                     # whole words, and element by element
def test_the_largest_values_take_the_code_below(fmt, dtype, H):
    big = torch.finfo(dtype).max
    x = torch.full((3, H), big, dtype=dtype)
    x[0, 1::2] *= -1
    # half a step above the top code; in int8 that is 127 * 2^121, which the next smaller exponent covers exactly, so that
    # every group with the top exponent has a value that would round up
    step = {"int8": 2.0 ** 122, "e4m3": 16 * 2.0 ** 120}[fmt]
    x[1] = TOP[fmt] + step / 2 if dtype == F32 else TOP[fmt]
    x[2] = TOP[fmt] / 2
    got = body.Act8Record(3, H, fmt).store(x.cuda()).load(dtype=F32).double().cpu()
    assert (got[0].abs() == TOP[fmt]).all() and torch.equal(got[0].sign(), x[0].double().sign())
    assert (got[1] == (127 * 2.0 ** 121 if fmt == "int8" and dtype == F32 else TOP[fmt])).all()
    want = O.record_values(x[2:].double().numpy(), fmt)     # further down nothing is special
    np.testing.assert_array_equal(got[2:].numpy(), want)
    assert (got[0].abs() - big).abs().max() <= step         # 2^128 is one step above the top code


def _tiny(T, H, seed):
    """Groups whose exponent is the smallest: values between 2^-133 and 2^-120 in size."""
    g = torch.Generator().manual_seed(seed)
    e = torch.randint(-133, -120, (T, H), generator=g).double()
    m = 1 + torch.rand(T, H, generator=g, dtype=torch.float64)
    s = torch.randint(0, 2, (T, H), generator=g).double() * 2 - 1
    return (s * m * 2.0 ** e).to(F32)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("H", [96, 95])
def test_the_smallest_exponent(fmt, H):
    x = _tiny(40, H, 1)
    rec = body.Act8Record(40, H, fmt).store(x.cuda())
    got = rec.load(dtype=F32).double().cpu().numpy()
    want = O.record_values(x.double().numpy(), fmt)
    np.testing.assert_array_equal(got, want)
    e, _ = O.record_exponents(x.double().numpy(), fmt)
    assert (e == -126).any()
    at = np.repeat(e == -126, 32, axis=1)[:, :H]
    err = np.abs(want - x.double().numpy())
    step = 2.0 ** -127 if fmt == "int8" else np.abs(x.double().numpy()) / 16 + 2.0 ** -136
    assert (err <= np.maximum(step, 0))[at].all()
    as_bf16 = rec.load(dtype=BF16)
    assert torch.equal(as_bf16.cpu(), torch.from_numpy(want).to(F32).to(BF16))
    if fmt == "int8":
        np.testing.assert_array_equal(as_bf16.double().cpu().numpy(), want)        # exact all the way down


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("T,N,H", [(40, 64, 96), (333, 136, 264), (40, 33, 65)])
def test_the_weight_gradient_at_the_smallest_exponent(fmt, T, N, H):
    """dY of 2^40 brings the results to fp32's normal range. Bounds as in the weight gradient's other tests: T 2^-24 + 2^-22
    of the sum of the terms' magnitudes."""
    x = _tiny(T, H, 2)
    rec = body.Act8Record(T, H, fmt).store(x.cuda())
    dy = (torch.randn(T, N, generator=torch.Generator().manual_seed(3)) * 2.0 ** 40).to(BF16)
    kept = O.record_values(x.double().numpy(), fmt)
    if N % 8 == 0 and H % 8 == 0:
        kept = torch.from_numpy(kept).to(F32).to(BF16).double().numpy()             # the operand that the tensor cores read
    got = body.Act8WeightGrad(T, N, H, dtype=F32).run(dy.cuda(), rec).double().cpu().numpy()
    d = dy.double().numpy()
    assert (np.abs(got - d.T @ kept) <= (T * 2.0 ** -24 + 2.0 ** -22) * (np.abs(d).T @ np.abs(kept))).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("T,N,H", [(40, 64, 96), (333, 136, 264), (40, 33, 65)])
def test_the_weight_gradient_across_exponents(fmt, T, N, H):
    """Groups from 2^-60 to 2^100 in size side by side, each group of columns of one size, so that the bound by the terms'
    magnitudes is that group's; dY of 2^-20. (An e4m3 operand's scale is split in two factors above 2^7.)"""
    g = torch.Generator().manual_seed(4)
    sizes = torch.tensor([2.0 ** e for e in (-60, -3, 0, 6, 8, 9, 30, 64, 100)])
    x = torch.randn(T, H, generator=g) * sizes[torch.arange(H) // 32 % len(sizes)]
    rec = body.Act8Record(T, H, fmt).store(x.cuda())
    dy = (torch.randn(T, N, generator=g) * 2.0 ** -20).to(BF16)
    kept, d = O.record_values(x.double().numpy(), fmt), dy.double().numpy()
    got = body.Act8WeightGrad(T, N, H, dtype=F32).run(dy.cuda(), rec).double().cpu().numpy()
    assert (np.abs(got - d.T @ kept) <= (T * 2.0 ** -24 + 2.0 ** -22) * (np.abs(d).T @ np.abs(kept))).all()
