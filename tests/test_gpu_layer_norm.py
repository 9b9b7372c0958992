"""Layer norm on the GPU against its formulas in 64 bits.

Tolerances: half a step of the output type relative to the value, and fp32 arithmetic: C = 64 units of 2^-24 of the terms
that an output is made of. (A row's mean and squares are sums of at most 8 values a thread and trip, five trips at the widest
row here, and ten levels of a tree: 50 additions; the few operations behind them make up the rest.) The error of the mean goes by
mean |x|, and with it that of xh by A = rho mean |x|. Column sums: one addition a row of a block and 64 in the join, N in all.
"""
import pytest
import torch

from paper_2608_03796_b200 import body
from paper_2608_03796_b200.autograd import act8_linear, layer_norm

pytestmark = pytest.mark.gpu
BF16, F16, F32, F64 = torch.bfloat16, torch.float16, torch.float32, torch.float64
UNIT, C = 2.0 ** -24, 64


def _step(t, dtype):
    return t.abs() * (torch.finfo(dtype).eps / 2) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def _near(got, want, slack, what):
    bad = (got.double() - want).abs() - (_step(want, got.dtype) + slack)
    assert torch.isfinite(got).all() and float(bad.max() if bad.numel() else -1) <= 0, f"{what}: {float(bad.max())} beyond the bound"


def _inputs(T, H, x_type, type, weight_type, seed=0, bias=True, pad=0, shift=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*s):
        return torch.randn(*s, generator=g, device="cuda")

    def placed(t):                                                          # rows apart, off a 16-byte boundary
        wide = torch.full((T, H + pad + shift), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, shift:shift + H] = t
        return wide[:, shift:shift + H]
    x = normal(T, H) * torch.exp(normal(H)) + normal(H)
    w, b = (1 + 0.3 * normal(H)).to(weight_type), (0.5 * normal(H)).to(weight_type) if bias else None
    return placed(x.to(x_type)), w, b, placed(normal(T, H).to(type))


def _check(x, w, b, dy, y, d, eps, stats, at=None):
    """`at`: where the backward pass takes x, if not at x (a record's values)."""
    T, H = x.shape
    X, W, D = x.double(), (torch.ones(H, device="cuda", dtype=F64) if w is None else w.double()), dy.double()
    mean = X.mean(1, keepdim=True)
    rho = ((X - mean).square().mean(1, keepdim=True) + eps) ** -0.5
    xh, A = (X - mean) * rho, rho * X.abs().mean(1, keepdim=True)
    want = xh * W + (0 if b is None else b.double())
    _near(y, want, C * UNIT * (W.abs() * (xh.abs() + A) + (0 if b is None else b.double().abs())), "y")
    if d is None:
        return
    if at is not None:
        mean, rho = stats[0].double()[:, None], stats[1].double()[:, None]
        X = at.double()
        xh, A = (X - mean) * rho, rho * X.abs().mean(1, keepdim=True)
    g = D * W
    m1, m2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    a1, a2 = g.abs().mean(1, keepdim=True), (g * xh).abs().mean(1, keepdim=True)
    slack = C * UNIT * rho * (g.abs() + a1 + xh.abs() * a2 + (xh.abs() + A) * (a2 + xh.abs() * a1) + A * a2)
    _near(d.x, rho * (g - m1 - xh * m2), slack, "dx")
    N = T / min(T, 148) + 80
    if w is not None:
        _near(d.weight, (D * xh).sum(0), UNIT * (N * (D * xh).abs().sum(0) + C * (D.abs() * (xh.abs() + A)).sum(0)), "dweight")
    if b is not None:
        _near(d.bias, D.sum(0), UNIT * N * D.abs().sum(0), "dbias")


# widths of a warp's rows, of a block's and wider ones, whole words and not; one row, fewer than blocks, more
@pytest.mark.parametrize("T,H", [(1, 1), (1, 8), (3, 256), (5, 257), (1000, 512), (1, 513), (7, 1000), (2, 2880), (1021, 2880),
                                 (700, 4096), (3, 4095), (2, 8192), (2, 8200), (333, 8201), (5, 40000)])
@pytest.mark.parametrize("type", [BF16, F32])
def test_against_the_formulas(T, H, type):
    x, w, b, dy = _inputs(T, H, type, type, type, seed=T + H)
    op = body.LayerNorm(T, H, dtype=type, eps=1e-5)
    y = op.forward(x, w, b)
    _check(x, w, b, dy, y, op.backward(dy), 1e-5, op.stats)


@pytest.mark.parametrize("x_type,type,weight_type", [(F16, F16, F16), (F32, BF16, BF16), (F32, F16, F32), (BF16, BF16, F32)])
@pytest.mark.parametrize("H", [200, 1000, 9000])
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 1)])
def test_types_strides_and_alignment(x_type, type, weight_type, H, pad, shift):
    T = 37
    x, w, b, dy = _inputs(T, H, x_type, type, weight_type, seed=H, pad=pad, shift=shift)
    op = body.LayerNorm(T, H, dtype=type, x_dtype=x_type, eps=1e-3)
    y = op.forward(x, w, b)
    _check(x, w, b, dy, y, op.backward(dy), 1e-3, op.stats)


@pytest.mark.parametrize("weight,bias", [(True, False), (False, True), (False, False)])
def test_without_weight_or_bias(weight, bias):
    x, w, b, dy = _inputs(50, 640, BF16, BF16, BF16)
    w, b = w if weight else None, b if bias else None
    op = body.LayerNorm(50, 640)
    y = op.forward(x, w, b)
    d = op.backward(dy)
    assert (d.weight is None) == (w is None) and (d.bias is None) == (b is None)
    _check(x, w, b, dy, y, d, 1e-5, op.stats)


@pytest.mark.parametrize("act8", ["int8", "e4m3"])
@pytest.mark.parametrize("T,H", [(9, 96), (65, 500), (40, 1000), (33, 2001), (3, 9001)])
def test_records(act8, T, H):
    """x's record is read in x's place; y's is that of y as it is returned."""
    x, w, b, dy = _inputs(T, H, BF16, BF16, BF16, seed=H)
    op = body.LayerNorm(T, H, act8=act8, keep_y=True)
    y = op.forward(x, w, b)
    for record, of in ((op.x_record, x), (op.y_record, y)):
        assert torch.equal(record.buffer[:T * ((H + 31) // 32 * 32)], body.Act8Record(T, H, act8).store(of).buffer[:T * ((H + 31) // 32 * 32)])
        assert torch.equal(record.load(dtype=F32), body.Act8Record(T, H, act8).store(of).load(dtype=F32))
    kept = op.x_record.load(dtype=F32)
    _check(x, w, b, dy, y, op.backward(dy), 1e-5, op.stats, at=kept)


@pytest.mark.parametrize("H", [300, 1024, 12000])
def test_variance_of_values_far_from_zero(H):
    """Values near 1000 whose spread is 1: a difference of sums of squares would lose the variance. xh is off by the mean's own
    rounding error at most, C units of 1000."""
    x, w, b, dy = _inputs(20, H, F32, F32, F32)
    x = 1000 + torch.randn(20, H, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    op = body.LayerNorm(20, H, dtype=F32)
    y = op.forward(x, w, b)
    _check(x, w, b, dy, y, op.backward(dy), 1e-5, op.stats)


def test_constant_rows_and_rows_that_are_not_finite():
    """A row of equal numbers has xh = 0 and y = bias, whatever its size; an infinity or a NaN spoils its own row and the
    column sums, and nothing else."""
    T, H = 6, 768
    x, w, b, dy = _inputs(T, H, BF16, BF16, BF16)
    x[1], x[2] = 3.0, 0.0
    x[4, 7] = float("inf")
    op = body.LayerNorm(T, H)
    y = op.forward(x, w, b)
    assert torch.equal(y[1], b) and torch.equal(y[2], b)
    assert not torch.isfinite(y[4]).any()
    d = op.backward(dy)
    fine = [0, 1, 2, 3, 5]
    assert torch.isfinite(y[fine]).all() and torch.isfinite(d.x[fine]).all() and not torch.isfinite(d.x[4]).any()


def test_no_rows():
    op = body.LayerNorm(0, 64)
    w = torch.ones(64, dtype=BF16, device="cuda")
    e = torch.empty(0, 64, dtype=BF16, device="cuda")
    assert op.forward(e, w, w).shape == (0, 64)
    d = op.backward(e)
    assert not d.weight.any() and not d.bias.any()


def test_results_are_the_same_every_time():
    x, w, b, dy = _inputs(2000, 1536, BF16, BF16, F32)
    op = body.LayerNorm(2000, 1536)
    first = [t.clone() for t in (op.forward(x, w, b), *op.backward(dy))]
    for _ in range(3):
        assert all(torch.equal(u, v) for u, v in zip(first, (op.forward(x, w, b), *op.backward(dy))))


def test_offsets_past_32_bits():
    T, H = (1 << 31) // 4096 + 40, 4096
    x = torch.zeros(T, H, dtype=BF16, device="cuda")
    tail, w, b, dy = _inputs(30, H, BF16, BF16, BF16)
    x[-30:] = tail
    op = body.LayerNorm(T, H)
    y = op.forward(x, w, b)
    _check(tail, w, b, dy, y[-30:], None, 1e-5, None)
    whole = torch.zeros(T, H, dtype=BF16, device="cuda")
    whole[-30:] = dy
    d = op.backward(whole)
    _check(tail, w, b, dy, y[-30:], d._replace(x=d.x[-30:]), 1e-5, None)


def test_captured_and_replayed_on_another_stream():
    T, H = 300, 1000
    x, w, b, dy = _inputs(T, H, BF16, BF16, BF16)
    op = body.LayerNorm(T, H)
    op.forward(x, w, b), op.backward(dy)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            y, d = op.forward(x, w, b), op.backward(dy)
        x.copy_(_inputs(T, H, BF16, BF16, BF16, seed=9)[0])
        for t in (y, *d):
            t.zero_()
        graph.replay()
    torch.cuda.synchronize()
    _check(x, w, b, dy, y, d, 1e-5, op.stats)


@pytest.mark.parametrize("act8", [None, "int8"])
def test_autograd(act8):
    """Leading dimensions, an input that is not contiguous, gradients of the right shapes; the record of y feeds act8_linear."""
    x, w, b, dy = _inputs(24, 320, BF16, BF16, BF16)
    lead = x.reshape(2, 12, 320).transpose(0, 1).requires_grad_()
    W = torch.randn(64, 320, device="cuda").to(BF16).requires_grad_()
    w.requires_grad_(), b.requires_grad_()
    if act8 is None:
        y = layer_norm(lead, w, b)
        (y * dy.reshape(2, 12, 320).transpose(0, 1)).sum().backward()
        rows = x.detach()
        _check(rows, w.detach(), b.detach(), dy, y.detach().transpose(0, 1).reshape(24, 320),
               body.LayerNormGrads(lead.grad.transpose(0, 1).reshape(24, 320), w.grad, b.grad), 1e-5, None)
    else:
        y, kept = layer_norm(lead, w, b, act8=act8, keep_y=True)
        act8_linear(y, W, record=kept).float().square().sum().backward()
        assert lead.grad.shape == lead.shape and W.grad.shape == W.shape and torch.isfinite(W.grad).all()
        with torch.no_grad():
            assert layer_norm(lead, w, b).shape == lead.shape


def test_refusals_on_the_device():
    op = body.LayerNorm(4, 64)
    x = torch.zeros(4, 64, dtype=BF16, device="cuda")
    w = torch.ones(64, dtype=BF16, device="cuda")
    for bad in (lambda: op.forward(x.float(), w), lambda: op.forward(x[:3], w), lambda: op.forward(x, w[:32]),
                lambda: op.forward(x, w, w.float()), lambda: op.forward(x.cpu(), w), lambda: op.forward(x.t().contiguous().t(), w)):
        with pytest.raises(TypeError):
            bad()
