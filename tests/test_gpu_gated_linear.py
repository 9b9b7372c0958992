"""The gated linear layer on the GPU against its formulas in 64 bits.

Tolerances. A product's sum over n terms is off by at most (n / 16 + 16) units of 2^-23 of the sum of the terms' magnitudes (the
tensor cores add 16 products at a time to an fp32 sum, each addition cutting at most a unit off; the kernel for few tokens adds
n / 64 of them a lane and joins 6 levels). With E that number and G, U the magnitudes of gate and up, h moves by
1.13 |u| E G + |act(g)| E U (|act'| <= 1.13), the backward values likewise (|act''| <= 1). act itself goes by exp(-|k|), k = g or
2 sqrt(2 / pi) (g + 0.044715 g^3): __expf is off by at most 2 + 1.173 |k| units of 2^-23 relative (CUDA's programming guide), k by
three roundings, which the exponential turns into 3 |k| / 2 units relative, quotient and products make up the rest of
S = (8 + 4 |k|) units. Every output adds half a step of its type. dx and the weight gradient are held against products of the dgate_up
that the call left, which is itself held against the formula.
"""
import math

import pytest
import torch

from paper_2608_03796_b200 import binding as B
from paper_2608_03796_b200 import body
from paper_2608_03796_b200.autograd import act8_linear, check_status, gated_act, gated_linear

pytestmark = pytest.mark.gpu
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def _act(act, x):
    """act(x) = x p and act'(x) = p + x p (1 - p) k', p = sigmoid(k), in 64 bits (1 + tanh would lose the far negative side)."""
    c = 2 * math.sqrt(2 / math.pi)
    k, slope = (x, 1.0) if act == "silu" else (c * (x + 0.044715 * x ** 3), c * (1 + 3 * 0.044715 * x * x))
    p = torch.sigmoid(k)
    return x * p, p + x * p * torch.sigmoid(-k) * slope


def _sigmoid_unit(act, g):
    k = g.abs() if act == "silu" else 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3).abs()
    return (8 + 4 * k) * 2.0 ** -23


def _unit(n):
    return (n / 16 + 16) * 2.0 ** -23


def _near(got, want, slack, what):
    t = torch.finfo(got.dtype)
    bad = (got.double() - want).abs() - (want.abs() * (t.eps / 2) + t.smallest_normal + slack)
    assert torch.isfinite(got).all() and (bad.numel() == 0 or float(bad.max()) <= 0), f"{what}: {float(bad.max())} beyond the bound"


def _inputs(T, H, F, seed=0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*s):
        return torch.randn(*s, generator=g, device="cuda")

    def apart(t):
        if not pad:
            return t
        wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, :t.shape[1]] = t
        return wide[:, :t.shape[1]]
    return apart(normal(T, H).to(BF16)), (1.5 * normal(2 * F, H) / H ** 0.5).to(BF16), apart((0.1 * normal(T, F)).to(BF16))


class _Want:
    def __init__(self, x, w, act):
        H, F = w.shape[1], w.shape[0] // 2
        X, W = x.double(), w.double()
        z, size = X @ W.t(), _unit(H) * (X.abs() @ W.abs().t())
        self.gate, self.up, self.dg, self.du = z[:, :F], z[:, F:], size[:, :F], size[:, F:]
        self.a, self.slope = _act(act, self.gate)
        self.h = self.a * self.up
        self.h_slack = 1.13 * self.up.abs() * self.dg + self.a.abs() * self.du + _sigmoid_unit(act, self.gate) * self.h.abs() + 1.13 * self.dg * self.du


def _check_back(op, x, w, dh, act, dx, dw, want, kept_x=None):
    """dgate_up against the formula at what was kept of gate and up, the two products against dgate_up."""
    F, D = op.F, dh.double()
    gate, up, dg, du = want.gate, want.up, want.dg, want.du
    if op.act8 is not None:
        gate, up, dg, du = op.gate_record.load(dtype=F32).double(), op.up_record.load(dtype=F32).double(), 0, 0
    a, slope = _act(act, gate)
    gelu = 2.0 ** -20 * (1 + gate.abs() if act == "gelu" else 1)            # the slope is a sum of terms of size 1 and |g|
    _near(op.dgate_up[:, :F], D * up * slope, D.abs() * (up.abs() * (dg + gelu) + 1.13 * du + dg * du), "dgate")
    _near(op.dgate_up[:, F:], D * a, D.abs() * (1.13 * dg + _sigmoid_unit(act, gate) * a.abs()), "dup")
    z, W, X = op.dgate_up.double(), w.double(), (x.double() if kept_x is None else kept_x.double())
    if dx is not None:
        _near(dx, z @ W, _unit(2 * F) * (z.abs() @ W.abs()), "dx")
    if dw is not None:
        _near(dw, z.t() @ X, _unit(len(x)) * (z.abs().t() @ X.abs()), "dweight")


# a token or two, up to 128 (each width of the narrow tile, its last columns empty or not), more
SHAPES = [(1, 8, 8), (1, 2048, 1000), (2, 72, 40), (3, 264, 136), (5, 4096, 264), (8, 1000, 128), (9, 64, 72), (16, 64, 64), (17, 2048, 72),
          (33, 1000, 1000), (64, 4096, 136), (65, 136, 12000), (128, 2816, 200), (129, 640, 200), (256, 512, 384), (300, 2816, 1416),
          (1021, 200, 2600)]


@pytest.mark.parametrize("T,H,F", SHAPES)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_nothing_kept(T, H, F, act):
    x, w, dh = _inputs(T, H, F, seed=T + H + F)
    op = body.GatedLinear(T, H, F, act=act)
    want = _Want(x, w, act)
    _near(op.forward(x, w), want.h, want.h_slack, "h")
    assert op.status()[0] == 0
    dx, dw = op.backward(dh)
    assert op.status()[0] == 0
    _check_back(op, x, w, dh, act, dx, dw, want)


@pytest.mark.parametrize("T,H,F", [(1, 64, 72), (7, 264, 136), (30, 136, 1000), (100, 512, 40), (300, 1024, 1416), (520, 72, 40)])
@pytest.mark.parametrize("act8", ["int8", "e4m3"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_records(T, H, F, act8, act):
    """Records of gate and up stand for them as closely as any record does, that of h for h as it was returned."""
    x, w, dh = _inputs(T, H, F, seed=T + F)
    op = body.GatedLinear(T, H, F, act=act, act8=act8, keep_h=True, dtype=F32)
    want = _Want(x, w, act)
    h = op.forward(x, w)
    _near(h, want.h, want.h_slack, "h")
    for record, z, slack in ((op.gate_record, want.gate, want.dg), (op.up_record, want.up, want.du)):
        rows = torch.nn.functional.pad(z.abs() + slack, (0, -F % 32)).reshape(T, -1, 32)
        top = rows.amax(-1, keepdim=True).expand(-1, -1, 32).reshape(T, -1)[:, :F]
        bound = top / 127 if act8 == "int8" else (z.abs() + slack) / 16 + top * 2.0 ** -17
        assert float(((record.load(dtype=F32).double() - z).abs() - bound - slack).max()) <= 0
    assert torch.equal(op.h_record.load(dtype=F32), body.Act8Record(T, F, act8).store(h).load(dtype=F32))
    Fp = (F + 31) // 32 * 32                                                # padding codes are zeros
    assert not op.gate_record.buffer[:T * Fp].view(T, Fp)[:, F:].any()
    record = body.Act8Record(T, H, act8).store(x)
    dx, dw = op.backward(dh, record)
    assert op.status()[0] == 0
    _check_back(op, x, w, dh, act, dx, dw, want, kept_x=record.load(dtype=F32))


def test_rows_apart_and_gradients_that_are_added():
    T, H, F = 70, 136, 264
    x, w, dh = _inputs(T, H, F, pad=8)
    for dtype in (BF16, F32):
        op = body.GatedLinear(T, H, F, dtype=dtype)
        want = _Want(x, w, "silu")
        _near(op.forward(x, w), want.h, want.h_slack, "h")
        dx, dw = op.backward(dh)
        _check_back(op, x, w, dh, "silu", dx, dw, want)
        total = torch.ones(2 * F, H, dtype=dtype, device="cuda")
        none, out = op.backward(dh, out=total, accumulate=True, want_dx=False)
        assert none is None and out is total
        z = op.dgate_up.double()
        _near(total, 1 + z.t() @ x.double(), _unit(T) * (z.abs().t() @ x.double().abs()) + 2.0 ** -23, "1 + dweight")
        assert op.backward(dh, want_dweight=False)[1] is None


@pytest.mark.parametrize("T,H,F", [(4096, 256, 128), (2000, 128, 128), (64, 4096, 2048)])
def test_long_contractions_with_few_tiles(T, H, F):
    """Their parts go through slabs in fp32, the last part shorter than the others."""
    x, w, dh = _inputs(T, H, F)
    op = body.GatedLinear(T, H, F)
    want = _Want(x, w, "silu")
    op.forward(x, w)
    first = [t.clone() for t in op.backward(dh)]
    _check_back(op, x, w, dh, "silu", *first, want)
    assert all(torch.equal(a, b) for a, b in zip(first, op.backward(dh)))


def test_rows_that_are_not_finite_stay_their_own():
    for T in (4, 40):
        x, w, dh = _inputs(T, 128, 256)
        x[1, 5], x[2, 7] = float("nan"), float("inf")
        h = body.GatedLinear(T, 128, 256).forward(x, w)
        fine = [t for t in range(T) if t not in (1, 2)]
        assert torch.isfinite(h[fine]).all() and torch.isnan(h[1]).all() and not torch.isfinite(h[2]).all()


def test_saturated_gates():
    """exp of a gate far out on either side: h is u g or 0, and the gradients are finite."""
    T, H, F = 16, 64, 64
    x = torch.zeros(T, H, dtype=BF16, device="cuda")
    x[:, 0] = torch.linspace(-300, 300, T).to(BF16).cuda()
    w = torch.ones(2 * F, H, dtype=BF16, device="cuda")
    for act in ("silu", "gelu"):
        op = body.GatedLinear(T, H, F, act=act)
        want = _Want(x, w, act)
        _near(op.forward(x, w), want.h, want.h_slack, "h")
        dx, dw = op.backward(torch.ones(T, F, dtype=BF16, device="cuda"))
        _check_back(op, x, w, torch.ones(T, F, device="cuda"), act, dx, dw, want)


def test_no_tokens():
    w = torch.ones(128, 64, dtype=BF16, device="cuda")
    e, d = torch.empty(0, 64, dtype=BF16, device="cuda"), torch.empty(0, 64, dtype=BF16, device="cuda")
    op = body.GatedLinear(0, 64, 64)
    assert op.forward(e, w).shape == (0, 64)
    dx, dw = op.backward(d)
    assert dx.shape == (0, 64) and not dw.any()


@pytest.mark.parametrize("act8", [None, "int8"])
def test_captured_and_replayed(act8):
    T, H, F = 200, 256, 384
    x, w, dh = _inputs(T, H, F)
    op = body.GatedLinear(T, H, F, act8=act8)
    record = None if act8 is None else body.Act8Record(T, H, act8).store(x)
    op.forward(x, w), op.backward(dh, record)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        if record is not None:
            record.store(x)
        h = op.forward(x, w)
        dx, dw = op.backward(dh, record)
    x.copy_(_inputs(T, H, F, seed=5)[0])
    graph.replay()
    torch.cuda.synchronize()
    want = _Want(x, w, "silu")
    _near(h, want.h, want.h_slack, "h")
    _check_back(op, x, w, dh, "silu", dx, dw, want, kept_x=None if record is None else record.load(dtype=F32))


@pytest.mark.parametrize("act8", [None, "int8", "e4m3"])
def test_autograd(act8):
    """Against differences of the formula in 64 bits, along a random direction of x and of the weight: the gradients' inner
    product with it. Off by the roundings' share (bf16: 2^-9 a factor, four of them, without preferred sign) and, from records,
    by theirs (int8 1/127 of a group's largest value, e4m3 1/16 of the value, at random)."""
    T, H, F = 96, 128, 160
    x, w, dh = _inputs(T, H, F)
    x, w = x.reshape(4, 24, H).requires_grad_(), w.requires_grad_()
    h = gated_linear(x, w, act="gelu", act8=act8)
    assert h.shape == (4, 24, F)
    h.backward(dh.reshape(4, 24, F))
    check_status()

    def total(a, b):
        z = a.reshape(T, H) @ b.t()
        return (_act("gelu", z[:, :F])[0] * z[:, F:] * dh.double()).sum()
    for t, other, grad in ((x, w, x.grad), (w, x, w.grad)):
        v = torch.randn(t.shape, dtype=F64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
        f = (lambda s: total(t.detach().double() + s * v, w.detach().double())) if t is x else \
            (lambda s: total(x.detach().double(), t.detach().double() + s * v))
        slope = float((f(1e-5) - f(-1e-5)) / 2e-5)
        spread = float(grad.double().norm())                                # the deviation of the inner product with a random v
        assert abs(float((grad.double() * v).sum()) - slope) <= (0.02 if act8 is None else 0.1) * spread


def test_a_block_of_a_student():
    """Its run with act8_linear behind it, records passed on, agrees with the two operators that it replaces."""
    T, H, F = 100, 256, 320
    x, w, _ = _inputs(T, H, F)
    down = (torch.randn(H, F, device="cuda") / F ** 0.5).to(BF16)
    grads = []
    for fused in (True, False):
        a, b, c = (t.clone().requires_grad_() for t in (x, w, down))
        kept_x = body.Act8Record(T, H, "int8").store(x)
        if fused:
            h, kept = gated_linear(a, b, act8="int8", record=kept_x, keep_h=True)
        else:
            h, kept = gated_act(act8_linear(a, b, record=kept_x), keep_h=True)
        act8_linear(h, c, record=kept).float().square().mean().backward()
        grads.append([t.grad.float() for t in (a, b, c)])
    check_status()
    for f, p in zip(*grads):       # the one rounds gate and up to 8 bits from fp32, the other from bf16: codes a step apart, rarely
        assert float((f - p).norm() / p.norm()) <= 0.02
    with torch.no_grad():
        assert torch.isfinite(gated_linear(x[:1], w)).all()
        assert gated_linear(x, w, act8="int8", keep_h=True)[1] is None


def test_refusals_on_the_device():
    T, H, F = 16, 64, 64
    x, w, dh = _inputs(T, H, F)
    op = body.GatedLinear(T, H, F, act8="int8")
    with pytest.raises(RuntimeError, match="before any forward"):
        op.backward(dh)
    op.forward(x, w)
    for bad in (lambda: op.forward(x.float(), w), lambda: op.forward(x, w[:F]), lambda: op.forward(x, torch.cat([w, w], 1)[:, :H]),
                lambda: op.backward(dh), lambda: op.backward(dh, body.Act8Record(T, H, "e4m3")),
                lambda: op.backward(dh, body.Act8Record(T, 32, "int8")), lambda: op.backward(dh.float(), body.Act8Record(T, H, "int8")),
                lambda: gated_linear(x, w, record=body.Act8Record(T, H, "int8"), act8="e4m3"), lambda: gated_linear(x, w[:, :32])):
        with pytest.raises(TypeError):
            bad()
    odd = torch.zeros(T, H + 4, dtype=BF16, device="cuda")[:, :H]           # rows off a 16-byte boundary
    with pytest.raises(B.KdklError):
        op.forward(odd, w)
    assert torch.isfinite(gated_linear(odd, w)).all()                       # autograd's entry copies such rows
