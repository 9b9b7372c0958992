"""Rotary positions on the GPU against the rotation in 64 bits.

Tolerance: half a step of the output type relative to the value, and C = 12 units of 2^-24 of m (|a| + |b|): the angle is
rounded once to fp32, as a number of half turns in [-1, 1] (2^-25 pi radians), sine and cosine to two units each, the factor
to one, and the two products and their sum take three more roundings.
"""
import math

import pytest
import torch

from paper_2608_03796_b200 import body
from paper_2608_03796_b200.autograd import rotary

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
UNIT, C = 2.0 ** -24, 12


def _turned(x, positions, D, R, layout, sign=1, base=10000.0, scaling="none", factor=1.0, length=0):
    """The rotation in 64 bits, and m (|a| + |b|) of every place."""
    i = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    if scaling == "ntk":
        base = base * factor ** (R / (R - 2))
    f, m = base ** (-2 * i / R), 1.0
    if scaling == "linear":
        f = f / factor
    if scaling == "yarn":
        k = ((length * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
        f, m = k * f + (1 - k) * f / factor, 0.1 * math.log(factor) + 1
    angle = sign * positions.double()[:, None, None] * f
    c, s = m * angle.cos(), m * angle.sin()
    x = x.double()
    first, second = (slice(0, R // 2), slice(R // 2, R)) if layout == "half" else (slice(0, R, 2), slice(1, R, 2))
    a, b = x[..., first], x[..., second]
    y, size = x.clone(), torch.zeros_like(x)
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    size[..., first] = size[..., second] = m * (a.abs() + b.abs())
    return y, size


def _near(got, want, size, what):
    t = torch.finfo(got.dtype)
    bad = (got.double() - want).abs() - (want.abs() * (t.eps / 2) + t.smallest_normal * t.eps + C * UNIT * size)
    assert torch.isfinite(got).all() and float(bad.max()) <= 0, f"{what}: {float(bad.max())} beyond the bound"


def _tensors(T, q, k, D, type, seed=0, extra=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(T, q + k + extra, D, generator=g, device="cuda").to(type)
    return x[:, :q], x[:, q:q + k]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("type", [BF16, F16, F32])
@pytest.mark.parametrize("T,q,k,D,R", [(1, 32, 8, 128, 128), (1, 1, 0, 2, 2), (7, 3, 1, 64, 32), (333, 4, 4, 96, 64), (2000, 8, 2, 80, 40),
                                       (1300, 5, 1, 128, 128), (50, 2, 2, 10, 6), (9, 1, 1, 1024, 1024), (40, 3, 3, 256, 4)])
def test_against_the_rotation(layout, type, T, q, k, D, R):
    xq, xk = _tensors(T, q, k, D, type, seed=T + D, extra=2)
    positions = torch.randint(0, 1 << 20, (T,), device="cuda")
    rope = body.Rotary(D, rotary_dim=R, layout=layout)
    for turn, sign in ((rope.forward, 1), (rope.backward, -1)):
        got = turn(xq, xk if k else None, positions)
        for y, x, name in zip(got, (xq, xk), "qk"):
            if y is None:
                continue
            _near(y, *_turned(x, positions, D, R, layout, sign), name)
            assert torch.equal(y[..., R:], x[..., R:])


@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 4.0), ("ntk", 8.0), ("yarn", 16.0)])
@pytest.mark.parametrize("wide", [torch.int32, torch.int64])
def test_scalings_and_far_positions(scaling, factor, wide):
    """Positions up to 2^30, negative ones too: their angles are exact to 2^-50 turns in 64 bits, here and in the oracle
    2^-53 of 2^28 turns: nothing beside the tolerance."""
    T, D = 256, 64
    far = torch.cat([torch.randint(-(1 << 30), 1 << 30, (T - 2,), device="cuda"), torch.tensor([0, 1], device="cuda")]).to(wide)
    xq, xk = _tensors(T, 2, 1, D, F32)
    args = dict(base=500000.0, scaling=scaling, factor=factor)
    rope = body.Rotary(D, original_length=2048, **args)
    for y, x in zip(rope.forward(xq, xk, far), (xq, xk)):
        _near(y, *_turned(x, far, D, D, "half", length=2048, **args), scaling)


def _view(how, T, heads, D, type):
    """A [T, heads, D] view of something larger and the memory that it is a view of."""
    if how == "heads first":
        mem = torch.full((heads, T, D), 7.0, dtype=type, device="cuda")
        return mem.transpose(0, 1), mem
    if how == "odd start":
        mem = torch.full((T * heads * D + 1,), 7.0, dtype=type, device="cuda")
        return mem[1:].view(T, heads, D), mem
    mem = torch.full((T, heads, D + 6), 7.0, dtype=type, device="cuda")
    return mem[..., 2:2 + D], mem


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("how", ["heads first", "odd start", "apart"])
@pytest.mark.parametrize("type", [BF16, F32])
def test_strides_and_given_outputs(layout, how, type):
    T, D, R = 21, 64, 48
    x, _ = _tensors(T, 3, 2, D, type)
    q, mem_q = _view(how, T, 3, D, type)
    out, mem = _view(how, T, 3, D, type)
    q.copy_(x)
    untouched = torch.ones_like(mem, dtype=torch.bool)
    positions = torch.arange(T, device="cuda") * 1000
    got, none = body.Rotary(D, rotary_dim=R, layout=layout).forward(q, None, positions, out=(out, None))
    assert got is out and none is None
    _near(out, *_turned(x, positions, D, R, layout), how)
    if how == "apart":                                                      # what lies between the heads stays as it was
        untouched[..., 2:2 + D] = False
    elif how == "odd start":
        untouched[1:] = False
    else:
        untouched[:] = False
    assert (mem[untouched] == 7).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_in_place(layout):
    T, D, R = 500, 128, 96
    xq, xk = _tensors(T, 4, 2, D, BF16)
    positions = torch.arange(T, device="cuda")
    rope = body.Rotary(D, rotary_dim=R, layout=layout)
    want = [t.clone() for t in rope.forward(xq, xk, positions)]
    q, k = xq.clone(), xk.clone()
    rope.forward(q, k, positions, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_there_and_back():
    """Forward, then backward with the same positions, is the identity times the square of the factor."""
    T, D = 100, 64
    xq, xk = _tensors(T, 2, 2, D, F32)
    positions = torch.arange(T, device="cuda") * 12345
    rope = body.Rotary(D, scaling="yarn", factor=4.0, original_length=4096)
    m2 = (0.1 * math.log(4.0) + 1) ** 2
    q, k = (t.clone() for t in rope.forward(xq, xk, positions))
    for back, x in zip(rope.backward(q, k, positions), (xq, xk)):
        size = x.abs().double()
        pair = size + size.roll(D // 2, dims=-1)
        assert float(((back.double() - m2 * x.double()).abs() - 4 * C * UNIT * m2 * pair).max()) <= 0


def test_no_tokens_and_one_tensor():
    rope = body.Rotary(64)
    e = torch.empty(0, 4, 64, dtype=BF16, device="cuda")
    q, k = rope.forward(e, e[:, :2], torch.empty(0, dtype=torch.int64, device="cuda"))
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)


def test_offsets_past_32_bits():
    T, heads, D = 70000, 256, 128                                           # 2.3 10^9 values
    x = torch.zeros(T, heads, D, dtype=BF16, device="cuda")
    x[-3:] = torch.randn(3, heads, D, device="cuda").to(BF16)
    positions = torch.arange(T, device="cuda")
    y, _ = body.Rotary(D).forward(x, None, positions)
    _near(y[-3:], *_turned(x[-3:], positions[-3:], D, D, "half"), "the last tokens")
    assert not y[:-3].any()


def test_autograd_and_capture():
    """Leading dimensions, gradients (a rotation's are its opposite), and a captured call that is replayed with new
    positions."""
    D = 64
    rope = body.Rotary(D, rotary_dim=32, layout="interleaved")
    q = torch.randn(2, 9, 4, D, device="cuda").requires_grad_()
    k = torch.randn(2, 9, 1, D, device="cuda").requires_grad_()
    positions = torch.arange(18, device="cuda").reshape(2, 9) * 7
    a, b = rotary(q, k, positions, rope)
    u, v = torch.randn_like(a), torch.randn_like(b)
    torch.autograd.backward([a, b], [u, v])
    flat = positions.reshape(-1)
    for got, x, name in ((a, q, "q"), (b, k, "k")):
        _near(got.detach().reshape(18, -1, D), *_turned(x.detach().reshape(18, -1, D), flat, D, 32, "interleaved"), name)
    for got, x, name in ((q.grad, u, "dq"), (k.grad, v, "dk")):
        _near(got.reshape(18, -1, D), *_turned(x.reshape(18, -1, D), flat, D, 32, "interleaved", sign=-1), name)
    k.grad = None
    rotary(q, k, positions, rope)[1].sum().backward()                       # one of the two without a gradient
    assert k.grad is not None and rotary(q, None, positions, rope).shape == q.shape

    x = torch.randn(18, 4, D, device="cuda")
    rope.forward(x, None, flat)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, _ = rope.forward(x, None, flat)
    flat += 100
    graph.replay()
    torch.cuda.synchronize()
    _near(y, *_turned(x, flat, D, 32, "interleaved"), "replayed")


def test_a_captured_call_keeps_its_outputs():
    """Calls of other shapes between replays take other buffers, and none is freed under the graph."""
    D, rope = 64, body.Rotary(64)
    x, n = torch.randn(3, 4, D, device="cuda"), torch.arange(3, device="cuda")
    rope.forward(x, None, n)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, _ = rope.forward(x, None, n)
    for T in (3, 500, 2):
        other = torch.randn(T, 4, D, device="cuda")
        z, _ = rope.forward(other, None, torch.arange(T, device="cuda"))
        fill = [torch.full((T, 4, D), 5.0, device="cuda") for _ in range(8)]
        want, n[0] = z.clone(), T
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, want) and all((f == 5).all() for f in fill)
        _near(y, *_turned(x, n, D, D, "half"), "replayed")


def test_refusals_on_the_device():
    rope = body.Rotary(64)
    x = torch.zeros(4, 2, 64, dtype=BF16, device="cuda")
    n = torch.arange(4, device="cuda")
    for bad in (lambda: rope.forward(x, x, n.float()), lambda: rope.forward(x, x, n.cpu()), lambda: rope.forward(x, x, n[:3]),
                lambda: rope.forward(x, x.float(), n), lambda: rope.forward(x[..., :32], x, n), lambda: rope.forward(x.cpu(), x, n),
                lambda: rope.forward(x, None, n, out=(x[:, :1], None)), lambda: rotary(x, x, n.reshape(2, 2), rope),
                lambda: rope.forward(torch.zeros(4, 64, 2, dtype=BF16, device="cuda").transpose(1, 2), None, n)):
        with pytest.raises(TypeError):
            bad()
