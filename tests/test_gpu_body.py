"""GPU parity of the student-body operators against the fp64 oracle, through the public classes and the C ABI.

Tolerances, from the arithmetic. Records are compared exactly: the scaling is by powers of two and the rounding is the
oracle's. Everything else is fp32 arithmetic on exact inputs, rounded once: U below is twice the half step of the output
type (2^-8 for bf16, 2^-10 for fp16, with the smallest subnormal as absolute floor; 0 for fp32), and the other half of it,
2^-9 or 2^-11, is far above the fp32 errors of a result that does not cancel. Where terms can cancel, the fp32 error goes
by the terms: ABS = 2e-5 of the sum of their magnitudes, about 300 fp32 roundings (a row sum is a tree of at most 32
serial terms a thread and 10 levels; exp and its quotient are good to a few 1e-7 relative). A sum over T products taken
one after the other is off by at most T 2^-24 of the sum of their magnitudes, tensor-core sums by less (16 products an
addition).
"""
import numpy as np
import pytest
import torch

from oracle import body_oracle as O
from paper_2608_03796_b200 import binding as B
from paper_2608_03796_b200 import body

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
U = {BF16: 2.0 ** -8, F16: 2.0 ** -10, F32: 0.0}
FLOOR = {BF16: 1e-38, F16: 2.0 ** -24, F32: 0.0}
ABS = 2e-5
NAN = float("nan")


def _dev():
    return torch.device("cuda:0")


def _randn(seed, *shape, dtype=BF16, scale=1.0, outliers=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, generator=g) * scale
    if outliers:
        x *= torch.exp(torch.randn(shape[-1], generator=g))
    return x.to(dtype)


def _np(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _placed(x, how):
    """x on the device: as it is, as columns of a wider tensor, or one element off a 16-byte boundary."""
    T, H = x.shape
    if how == "plain":
        return x.to(_dev())
    if how == "wide":
        w = torch.full((T, 2 * H + 8), NAN, dtype=x.dtype, device=_dev())
        w[:, 8:8 + H] = x.to(_dev())
        return w[:, 8:8 + H]
    w = torch.full((T, H + 3), NAN, dtype=x.dtype, device=_dev())
    w[:, 1:1 + H] = x.to(_dev())
    return w[:, 1:1 + H]


def _close(got, want, dtype, terms=0.0, what=""):
    got, want = _np(got) if isinstance(got, torch.Tensor) else got, np.asarray(want)
    assert got.shape == want.shape, (got.shape, want.shape)
    err = np.abs(got - want) - (U[dtype] * np.abs(want) + FLOOR[dtype] + ABS * terms)
    assert np.isfinite(got).all(), what
    worst = np.unravel_index(np.argmax(err), err.shape)
    assert (err <= 0).all(), f"{what}: at {worst} {got[worst]} against {want[worst]}, {int((err > 0).sum())} places"


# ------------------------------------------------------------------ records

SHAPES = [(1, 1), (1, 4096), (3, 31), (5, 32), (7, 33), (37, 72), (130, 1000), (9, 2816), (33, 2049), (2, 4100), (400, 264)]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("how", ["plain", "wide", "odd"])
def test_record_is_the_oracles(fmt, dtype, how):
    for T, H in SHAPES:
        x = _randn(T * 7 + H, T, H, dtype=dtype, outliers=True)
        if H > 40 and T > 2:
            x[1, 2:34] = 0.0
            x[2] *= 1e-4 if dtype == F16 else 1e-30
        want = O.record_values(_np(x), fmt)
        rec = body.Act8Record(T, H, fmt)
        guard = torch.full((rec.nbytes + 512,), 0x5A, dtype=torch.uint8, device=_dev())   # nothing past the record
        rec.buffer, rec.ptr = guard[:rec.nbytes], guard.data_ptr()
        rec.store(_placed(x, how))
        assert (guard[rec.nbytes:] == 0x5A).all()
        got = rec.load(dtype=F32)
        np.testing.assert_array_equal(_np(got), want)
        assert np.array_equal(_np(rec.load(dtype=BF16)), want) or dtype == F32      # exact in bf16 but for subnormals
        out = _placed(torch.zeros(T, H, dtype=F32), how)
        base = out._base if out._base is not None else out
        before = base.clone()
        rec.load(out)
        np.testing.assert_array_equal(_np(out), want)
        mask = torch.ones_like(base, dtype=torch.bool)
        if base is not out:
            off = 8 if how == "wide" else 1
            mask[:, off:off + H] = False
            same = (base == before) | (base.isnan() & before.isnan())
            assert same[mask].all()
        # keeping what a record stands for changes nothing
        again = body.Act8Record(T, H, fmt).store(got).load(dtype=F32)
        assert torch.equal(again, got)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_record_of_extremes(fmt):
    big = torch.finfo(BF16).max
    x = torch.zeros(8, 96, dtype=BF16)
    x[0, 0] = float("inf"); x[0, 40] = 3.0
    x[1, 33] = NAN; x[1, 0] = -2.0
    x[2, :] = big; x[2, 1] = -big                       # rounding up would pass the largest finite number
    x[3, :] = torch.finfo(BF16).tiny                     # smallest normal
    x[4, :] = 2.0 ** -133                                # smallest subnormal
    x[5, :] = -0.0
    x[6, ::2] = 1.0; x[6, 1::2] = 2.0 ** -20             # far below the group's step
    rec = body.Act8Record(8, 96, fmt).store(x.to(_dev()))
    got = _np(rec.load(dtype=F32))
    assert np.isnan(got[0, :32]).all() and np.isfinite(got[0, 32:]).all() and abs(got[0, 40] - 3.0) <= 3.0 / 16
    assert np.isnan(got[1, 32:64]).all() and np.isfinite(got[1, :32]).all() and np.isfinite(got[1, 64:]).all()
    assert np.isfinite(got[2]).all() and (np.abs(got[2]) >= 0.9 * big).all() and got[2, 1] < 0
    np.testing.assert_array_equal(got[3:], O.record_values(_np(x)[3:], fmt))
    y = torch.full((1, 32), 65504.0, dtype=F16, device=_dev())
    back = body.Act8Record(1, 32, fmt).store(y).load(dtype=F16)
    assert torch.isfinite(back).all() and (back >= 0.9 * 65504).all()


# ------------------------------------------------------------------ gated activation


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype,fmt", [(BF16, "int8"), (BF16, "e4m3"), (F16, "e4m3"), (F16, "int8"), (BF16, None)])
@pytest.mark.parametrize("T,F,how", [(1, 8, "plain"), (1, 7168, "halves"), (3, 31, "plain"), (130, 264, "halves"),
                                     (33, 1001, "halves"), (9, 2816, "odd"), (257, 4100, "wide")])
def test_gated_matches_oracle(act, dtype, fmt, T, F, how):
    g, u = _randn(T + F, T, F, dtype=dtype, scale=3.0), _randn(T + F + 1, T, F, dtype=dtype)
    g[0, 0], u[0, 0] = 0.0, 0.0
    if F > 40:
        g[0, 1], g[0, 2] = 60.0, -60.0                    # a sigmoid that has saturated on either side
    dh = _randn(T + F + 2, T, F, dtype=dtype, scale=0.1)
    if how == "halves":
        both = torch.cat([g, u], 1).to(_dev())
        gd, ud = both[:, :F], both[:, F:]
    else:
        gd, ud = _placed(g, how), _placed(u, how)
    op = body.GatedAct(T, F, act=act, act8=fmt, dtype=dtype, keep_h=fmt is not None)
    op.h.fill_(NAN)
    h = op.forward(gd, ud)
    assert h is op.h
    _close(h, O.gated_forward(_np(g), _np(u), act), dtype, 0.0, "h")
    if fmt is None:
        with pytest.raises(RuntimeError):
            op.backward(dh.to(_dev()))
        return
    np.testing.assert_array_equal(_np(op.h_record.load(dtype=F32)), O.record_values(_np(h), fmt))
    gk, uk = O.record_values(_np(g), fmt), O.record_values(_np(u), fmt)
    np.testing.assert_array_equal(_np(op.gate_record.load(dtype=F32)), gk)
    np.testing.assert_array_equal(_np(op.up_record.load(dtype=F32)), uk)
    dg, du = op.backward(_placed(dh, "plain" if how == "halves" else how))
    want_g, want_u = O.gated_backward(gk, uk, _np(dh), act)
    _close(dg, want_g, dtype, np.abs(_np(dh) * uk) * (1 + np.abs(gk)), "dgate")     # act' has a zero: two terms cancel
    _close(du, want_u, dtype, 0.0, "dup")


def test_gated_derivative_is_the_forward_kernels():
    """Central differences of the forward kernel itself along the gradient. With steps of 2^-4 the fp16 rounding of h
    (2^-12 relative a value) averages out over 131072 values to below 1e-4 of the derivative, and the step's own
    error is of the order of (2^-4)^2 times a third derivative near 1: 2 % covers both."""
    T, F, step = 256, 512, 2.0 ** -4
    g, u = _randn(1, T, F, dtype=F16).to(_dev()), _randn(2, T, F, dtype=F16).to(_dev())
    for act in ("silu", "gelu"):
        op = body.GatedAct(T, F, act=act, act8="int8", dtype=F16)
        g8 = body.Act8Record(T, F).store(g).load(dtype=F16)
        u8 = body.Act8Record(T, F).store(u).load(dtype=F16)
        op.forward(g8, u8)
        dh = _randn(3, T, F, dtype=F16).to(_dev())
        dg, du = (t.double() for t in op.backward(dh))
        for grad, which in ((dg, 0), (du, 1)):
            v = (grad.sign() * step).half()
            plus = op.forward(*((g8 + v, u8) if which == 0 else (g8, u8 + v))).double().clone()
            minus = op.forward(*((g8 - v, u8) if which == 0 else (g8, u8 - v))).double().clone()
            diff = (dh.double() * (plus - minus)).sum().item() / 2
            want = (grad * v.double()).sum().item()
            assert abs(diff - want) <= 0.02 * abs(want), (act, which, diff, want)


# ------------------------------------------------------------------ weight gradient


DW_SHAPES = [(1, 8, 8), (1, 64, 4096), (16, 72, 40), (65, 256, 256), (333, 136, 520), (700, 1000, 264), (1030, 512, 1032),
             (130, 33, 65), (130, 136, 65), (130, 33, 64)]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("how", ["plain", "wide", "odd"])
def test_dweight_matches_oracle(fmt, dtype, how):
    for T, N, H in DW_SHAPES:
        dy, x = _randn(T + N, T, N), _randn(T + H, T, H, outliers=True)
        rec = body.Act8Record(T, H, fmt).store(x.to(_dev()))
        xk = O.record_values(_np(x), fmt)
        want = O.dweight(_np(dy), xk)
        terms = np.abs(_np(dy)).T @ np.abs(xk)
        op = body.Act8WeightGrad(T, N, H, dtype=dtype)
        op.dweight.fill_(NAN)
        dyd = _placed(dy, how)
        got = op.run(dyd, rec).clone()
        bound = (T * 2.0 ** -24 + 2.0 ** -22) / ABS * terms
        _close(got, want, dtype, bound, f"dW {(T, N, H)}")
        assert torch.equal(op.run(dyd, rec), got)                           # bit for bit
        base = _randn(9, N, H, dtype=dtype).to(_dev())
        out = base.clone()
        op.run(dyd, rec, out=out, accumulate=True)
        _close(out, _np(base) + want, dtype, bound + np.abs(_np(base)) * 2.0 ** -22 / ABS, f"dW += {(T, N, H)}")
        assert op.status()[0] == 0


@pytest.mark.parametrize("T,N,H,dtype", [(6000, 264, 520, F32), (6000, 264, 520, BF16), (20000, 64, 96, F32),
                                         (2500, 1000, 1544, BF16), (1536, 2048, 2560, F32)])
def test_dweight_over_long_batches(T, N, H, dtype):
    """Many runs of an accumulator, contractions in several parts, parts and runs of uneven length, several tiles a CTA
    pair. Against float64 on the GPU, with the bound of the tests above."""
    dy, x = _randn(1, T, N).to(_dev()), _randn(2, T, H, outliers=True).to(_dev())
    rec = body.Act8Record(T, H).store(x)
    xk = rec.load(dtype=F32).double()
    op = body.Act8WeightGrad(T, N, H, dtype=dtype)
    op.dweight.fill_(NAN)
    op.workspace.fill_(0xFF)
    got = op.run(dy, rec)
    terms = _np(dy.double().abs().t() @ xk.abs())
    _close(got, _np(dy.double().t() @ xk), dtype, (T * 2.0 ** -24 + 2.0 ** -22) / ABS * terms)
    want = got.clone()
    op.workspace.fill_(0xFF)
    assert torch.equal(op.run(dy, rec), want) and op.status()[0] == 0


def test_dweight_of_records_that_are_not_finite_and_of_nothing():
    T, N, H = 100, 64, 256
    x = _randn(1, T, H); x[50, 70] = float("inf")
    dy = _randn(2, T, N)
    rec = body.Act8Record(T, H).store(x.to(_dev()))
    op = body.Act8WeightGrad(T, N, H, dtype=F32)
    got = _np(op.run(dy.to(_dev()), rec))
    assert np.isnan(got[:, 64:96]).all()                                    # the group's columns say so ...
    rest = np.r_[0:64, 96:H]
    assert np.isfinite(got[:, rest]).all()                                  # ... and no others
    for T in (0,):
        rec = body.Act8Record(T, H)
        op = body.Act8WeightGrad(T, N, H, dtype=F32)
        op.dweight.fill_(NAN)
        op.run(torch.empty(0, N, dtype=BF16, device=_dev()), rec)
        assert not op.dweight.any()
        op.dweight.fill_(2.0)
        op.run(torch.empty(0, N, dtype=BF16, device=_dev()), rec, accumulate=True)
        assert (op.dweight == 2.0).all()


# ------------------------------------------------------------------ block norm


def _norm_case(T, H, dtype, rdtype, wdtype, kind, post, pre, fmt, how, with_dsum=True, offset=0.0, alpha=0.75, beta=0.9):
    eps = 1e-5
    r, b = _randn(1, T, H, dtype=rdtype, outliers=True), _randn(2, T, H, dtype=dtype)
    w1 = (1 - offset + 0.2 * _randn(3, H, dtype=F32)).to(wdtype) if post else None
    w2 = (1 - offset + 0.2 * _randn(4, H, dtype=F32)).to(wdtype) if pre else None
    gate = None if kind == "none" else (0.5 + 0.5 * _randn(5, H if kind == "channel" else T, dtype=F32)).to(wdtype)
    if gate is not None:
        gate[0] = 0.0                                                       # a closed gate still has a gradient
    dy, dx = _randn(6, T, H, dtype=dtype), _randn(7, T, H, dtype=rdtype)
    up = lambda t: None if t is None else t.to(_dev())                      # noqa: E731
    op = body.BlockNorm(T, H, dtype=dtype, residual_dtype=rdtype, gate=kind, act8=fmt, eps=eps, weight_offset=offset,
                        branch_scale=alpha, residual_scale=beta, keep_y=fmt is not None and pre)
    for t in (op.y, op.sum, op.rho):
        t.fill_(NAN)
    y, x = op.forward(_placed(r, how), _placed(b, how), post_weight=up(w1), pre_weight=up(w2), gate=up(gate))
    nps = lambda t: None if t is None else _np(t)                           # noqa: E731
    args = dict(w1=nps(w1), w2=nps(w2), gate=nps(gate), kind=kind, offset=offset, alpha=alpha, beta=beta)
    f = O.norm_forward(_np(r), _np(b), eps=eps, **args)
    into = np.abs(beta * _np(r)) + np.abs(f["x"] - beta * _np(r))
    _close(x, f["x"], rdtype, into, "x")
    if pre:
        _close(y, f["y"], dtype, into * np.abs(f["rho2"] * (_np(w2) + offset)), "y")
    else:
        assert y is None
    bk, xk = _np(b), _np(x)
    if fmt is not None:
        bk, xk = O.record_values(bk, fmt), O.record_values(xk, fmt)
        np.testing.assert_array_equal(_np(op.branch_record.load(dtype=F32)), bk)
        np.testing.assert_array_equal(_np(op.sum_record.load(dtype=F32)), xk)
        if pre:
            np.testing.assert_array_equal(_np(op.y_record.load(dtype=F32)), O.record_values(_np(y), fmt))
    d = op.backward(_placed(dy, how) if pre else None, _placed(dx, how) if with_dsum else None)
    o = O.norm_backward(_np(dy) if pre else None, _np(dx) if with_dsum else None, bk, xk, f["rho1"], f["rho2"], **args)
    # magnitudes of the terms that add up to each result
    md = np.abs(_np(dx)) if with_dsum else np.zeros((T, H))
    if pre:
        gy, xh = np.abs(_np(dy) * (_np(w2) + offset)), np.abs(xk * f["rho2"])
        md = md + f["rho2"] * (gy + xh * (gy * xh).mean(1, keepdims=True))
        _close(d.pre_weight, o["dw2"], wdtype, (np.abs(_np(dy)) * xh).sum(0), "dpre_weight")
    else:
        assert d.pre_weight is None
    _close(d.residual, o["dr"], rdtype, np.abs(beta) * md, "dresidual")
    k = np.abs(alpha * (1.0 if kind == "none" else _np(gate)[:, None] if kind == "token" else _np(gate)[None, :]))
    bh, w = np.abs(bk * f["rho1"]), (np.abs(_np(w1) + offset) if post else 1.0)
    mb = k * md * w
    if post:
        mb = f["rho1"] * (mb + bh * (mb * bh).mean(1, keepdims=True))
        _close(d.post_weight, o["dw1"], wdtype, (k * md * bh).sum(0), "dpost_weight")
    else:
        assert d.post_weight is None
    _close(d.branch, o["db"], dtype, mb, "dbranch")
    if kind != "none":
        _close(d.gate, o["dgate"], wdtype, (np.abs(alpha) * md * bh * w).sum(1 if kind == "token" else 0), "dgate")
    first = [t.clone() for t in d if t is not None]
    op.workspace.fill_(0xFF)
    again = op.backward(_placed(dy, how) if pre else None, _placed(dx, how) if with_dsum else None)
    assert all(torch.equal(s, t) for s, t in zip(first, (t for t in again if t is not None)))    # bit for bit


@pytest.mark.parametrize("T,H,how", [(1, 8, "plain"), (1, 4096, "plain"), (5, 33, "plain"), (37, 72, "wide"), (130, 1024, "plain"),
                                     (9, 1030, "odd"), (33, 2816, "wide"), (40, 4096, "odd"), (700, 96, "plain"),
                                     (1300, 264, "plain"), (6, 8192, "plain"), (5, 8200, "plain"), (3, 16384, "plain"),
                                     (3, 32768, "plain"), (2, 20001, "plain")])
@pytest.mark.parametrize("kind,fmt", [("none", None), ("channel", "int8"), ("token", "e4m3"), ("channel", None)])
def test_norm_matches_oracle(T, H, how, kind, fmt):
    _norm_case(T, H, BF16, BF16, BF16, kind, True, True, fmt, how)


@pytest.mark.parametrize("post,pre", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("kind", ["none", "channel", "token"])
@pytest.mark.parametrize("fmt", [None, "int8"])
def test_norm_parts_may_be_absent(post, pre, kind, fmt):
    _norm_case(50, 520, BF16, BF16, F32, kind, post, pre, fmt, "plain")


@pytest.mark.parametrize("dtype,rdtype,wdtype", [(BF16, F32, F32), (F16, F16, F16), (F16, F32, BF16), (BF16, BF16, F16)])
@pytest.mark.parametrize("fmt", [None, "int8", "e4m3"])
def test_norm_types(dtype, rdtype, wdtype, fmt):
    _norm_case(70, 1032, dtype, rdtype, wdtype, "channel", True, True, fmt, "plain", offset=1.0)
    _norm_case(70, 1000, dtype, rdtype, wdtype, "token", True, True, fmt, "odd", with_dsum=False, alpha=-1.5, beta=0.0)


@pytest.mark.parametrize("T,H", [(20, 8192), (5, 4104), (9, 12288), (7, 16392), (3, 32768)])
@pytest.mark.parametrize("fmt", [None, "int8"])
def test_norm_wide_rows(T, H, fmt):
    """An fp32 residual stream at the widths that need most shared memory, and rows shared by two and four blocks."""
    _norm_case(T, H, BF16, F32, F32, "channel", True, True, fmt, "plain")
    _norm_case(T, H, F16, F16, F32, "token", True, False, fmt, "plain", with_dsum=True)
    _norm_case(T, H, BF16, BF16, F32, "none", False, True, fmt, "wide", with_dsum=False)


def test_norm_of_zero_rows_and_of_a_sum_that_cancels():
    """A row of zeros has rho = eps^-1/2 and finite results; a residual that the branch cancels exactly gives y = 0."""
    T, H, eps = 4, 256, 1e-5
    b = _randn(1, T, H); b[1] = 0
    r = _randn(2, T, H); r[1] = 0
    op = body.BlockNorm(T, H, eps=eps)
    w = torch.ones(H, dtype=BF16, device=_dev())
    y, x = op.forward(r.to(_dev()), b.to(_dev()), post_weight=w, pre_weight=w)
    assert not y[1].any() and not x[1].any()
    d = op.backward(_randn(3, T, H).to(_dev()), None)
    assert all(torch.isfinite(t).all() for t in d if t is not None)
    op = body.BlockNorm(T, H, eps=eps, branch_scale=-1.0)
    y, x = op.forward(b.to(_dev()), b.to(_dev()), pre_weight=w)
    assert not x.any() and not y.any()
    d = op.backward(_randn(3, T, H).to(_dev()), None)
    assert torch.isfinite(d.branch).all() and torch.isfinite(d.residual).all()


def test_norm_nan_stays_in_its_row():
    T, H = 6, 512
    r, b = _randn(1, T, H), _randn(2, T, H)
    b[3, 17] = NAN
    w = torch.ones(H, dtype=BF16, device=_dev())
    op = body.BlockNorm(T, H, act8="int8")
    y, x = op.forward(r.to(_dev()), b.to(_dev()), post_weight=w, pre_weight=w)
    keep = [0, 1, 2, 4, 5]
    assert torch.isnan(y[3]).all() and torch.isfinite(y[keep]).all()
    d = op.backward(_randn(3, T, H).to(_dev()), _randn(4, T, H).to(_dev()))
    assert torch.isfinite(d.branch[keep]).all() and torch.isfinite(d.residual[keep]).all() and torch.isnan(d.branch[3]).all()


# ------------------------------------------------------------------ streams, graphs, launches, nothing to do


def test_other_stream_and_graph_replay():
    """Calls go to the current stream and can be captured: a replay on new inputs gives what the calls give."""
    T, H, N = 300, 512, 256
    dev = _dev()
    r, b, dy, dx = (_randn(s, T, H).to(dev) for s in range(4))
    w = (1 + 0.1 * _randn(9, H, dtype=F32)).to(BF16).to(dev)
    join = body.BlockNorm(T, H, act8="int8", keep_y=True)
    grad = body.Act8WeightGrad(T, N, H)
    ffn = body.GatedAct(T, N)
    dz = _randn(11, T, N).to(dev)

    def step():
        y, x = join.forward(r, b, post_weight=w, pre_weight=w)
        h = ffn.forward(y[:, :N], x[:, :N])
        d = join.backward(dy, dx)
        return [y, x, h, d.branch, d.residual, d.pre_weight, grad.run(dz, join.y_record), *ffn.backward(dz)]
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for t, s in ((r, 20), (b, 21), (dy, 22), (dx, 23), (dz, 24)):
        t.copy_(_randn(s, *t.shape))
    graph.replay()
    got = [t.clone() for t in outs]
    assert all(torch.equal(a, c) for a, c in zip(got, step()))
    assert not torch.equal(got[0], want[0])


def test_odd_addresses():
    """Vectors and results that do not start on 16 or 32 bytes take the element-wise paths and give the same."""
    T, H, N = 40, 264, 72
    dev = _dev()

    def off(t, by):                                                         # the same values, `by` elements off the boundary
        base = torch.empty(t.numel() + 64, dtype=t.dtype, device=dev)
        v = base[by:by + t.numel()].view(t.shape)
        return v.copy_(t.to(dev))
    r, b, dy, dx = (_randn(s, T, H) for s in range(4))
    w, gate = (1 + 0.1 * _randn(5, H, dtype=F32)), (1 + 0.1 * _randn(6, H, dtype=F32))
    results = []
    for by_w, by_x in ((0, 0), (4, 0), (1, 0), (0, 8), (0, 3)):             # fp32: 16 and 4 bytes off; bf16: 16 and 6
        op = body.BlockNorm(T, H, gate="channel", residual_dtype=F32)
        y, x = op.forward(off(r.float(), by_w), off(b, by_x), off(w, by_w), off(w, by_w), off(gate, by_w))
        d = op.backward(off(dy, by_x), off(dx.float(), by_w))
        results.append([t.clone().double() for t in (y, x, *d)])
    for other in results[1:]:
        for s, t in zip(results[0], other):
            assert ((s - t).norm() / s.norm()).item() <= 1e-3               # the same but for roundings at the last place
    rec = body.Act8Record(T, H).store(off(r, 0))
    want = body.Act8WeightGrad(T, N, H, dtype=F32).run(off(_randn(9, T, N), 0), rec)
    for by in (4, 1):
        out = off(torch.zeros(N, H), by)
        body.Act8WeightGrad(T, N, H, dtype=F32).run(off(_randn(9, T, N), 0), rec, out=out)
        assert ((out - want).norm() / want.norm()).item() <= 1e-5
        for dtype in (F32, BF16):
            x = _randn(11, T, H, dtype=dtype)
            a = body.Act8Record(T, H).store(off(x, by)).load(off(torch.zeros(T, H, dtype=dtype), by))
            assert torch.equal(a, body.Act8Record(T, H).store(off(x, 0)).load(dtype=dtype))


def test_offsets_past_32_bits():
    """A record of more than 2^32 codes, read and written to its end; the weight gradient over it."""
    T, H, N = (1 << 20) + 77, 4128, 16
    x = torch.empty(T, H, dtype=BF16, device=_dev())
    g = torch.Generator(device=_dev()).manual_seed(1)
    for t in range(0, T, 1 << 17):
        x[t:t + (1 << 17)].normal_(generator=g)
    rec = body.Act8Record(T, H).store(x)
    assert rec.nbytes > 1 << 32
    last = body.Act8Record(1000, H).store(x[-1000:]).load()
    out = torch.empty_like(x)
    rec.load(out)
    assert torch.equal(out[-1000:], last)
    assert torch.equal(out[:1000], body.Act8Record(1000, H).store(x[:1000]).load())
    dy = _randn(3, T, N, scale=0.1).to(_dev())
    got = body.Act8WeightGrad(T, N, H, dtype=F32).run(dy, rec)
    want = torch.zeros(N, H, dtype=torch.float64, device=_dev())
    for t in range(0, T, 1 << 17):
        want += dy[t:t + (1 << 17)].double().t() @ out[t:t + (1 << 17)].double()
    assert ((got.double() - want).norm() / want.norm()).item() <= 1e-5
    op = body.BlockNorm(T, H, act8="int8")
    w = torch.ones(H, dtype=BF16, device=_dev())
    y, s = op.forward(x, x, w, w)
    tail = body.BlockNorm(1000, H, act8="int8")
    y2, s2 = tail.forward(x[-1000:], x[-1000:], w, w)
    assert torch.equal(y[-1000:], y2) and torch.equal(s[-1000:], s2)
    d, d2 = op.backward(x, x), tail.backward(x[-1000:], x[-1000:])
    assert torch.equal(d.branch[-1000:], d2.branch) and torch.equal(d.residual[-1000:], d2.residual)


def test_refusals_of_tensors():
    """What a class was not made for is refused before anything is launched: types, shapes, strides, gates."""
    T, H = 8, 64
    dev = _dev()
    x = _randn(1, T, H).to(dev)
    w = torch.ones(H, dtype=BF16, device=dev)
    rec = body.Act8Record(T, H).store(x)
    for bad in (x.t(), x[:4], x.long(), x[:1].expand(T, H), x.cpu(), x.reshape(-1)):
        with pytest.raises((TypeError, ValueError)):
            rec.store(bad)
        with pytest.raises((TypeError, ValueError)):
            rec.load(bad)
    ffn = body.GatedAct(T, H)
    with pytest.raises(TypeError):
        ffn.forward(x, x.half())
    with pytest.raises(TypeError):
        ffn.forward(x, torch.cat([x, x], 1)[:, :H])                         # rows not equally far apart
    grad = body.Act8WeightGrad(T, 32, H)
    with pytest.raises(TypeError):
        grad.run(_randn(2, T, 32, dtype=F32).to(dev), rec)
    with pytest.raises(TypeError):
        grad.run(_randn(2, T, 32).to(dev), body.Act8Record(T, 32))
    with pytest.raises(TypeError):
        grad.run(_randn(2, T, 32).to(dev), rec, out=torch.empty(32, H, device=dev))
    join = body.BlockNorm(T, H, gate="token")
    with pytest.raises(TypeError):
        join.forward(x, x, w, w)                                            # the gate is missing
    with pytest.raises(TypeError):
        join.forward(x, x, w, w, gate=w)                                    # one per channel, not per token
    with pytest.raises(TypeError):
        join.forward(x, x, w, w.float(), gate=w[:T])                        # two weight types
    join.forward(x, x, w, None, gate=w[:T].clone())
    with pytest.raises(TypeError):
        join.backward(x, x)                                                 # there is no y
    with pytest.raises(TypeError):
        body.Act8Record(T, H, buffer=torch.empty(16, dtype=torch.uint8, device=dev))
    with pytest.raises(RuntimeError):
        body.BlockNorm(T, H, train=False).backward(x, x)


def test_no_tokens():
    dev = _dev()
    e = torch.empty(0, 64, dtype=BF16, device=dev)
    w = torch.ones(64, dtype=BF16, device=dev)
    body.Act8Record(0, 64).store(e).load()
    op = body.GatedAct(0, 64)
    assert op.forward(e, e).shape == (0, 64) and op.backward(e)[0].shape == (0, 64)
    join = body.BlockNorm(0, 64, act8="int8", gate="channel")
    y, x = join.forward(e, e, post_weight=w, pre_weight=w, gate=w)
    d = join.backward(e, e)
    assert y.shape == (0, 64) and not d.post_weight.any() and not d.pre_weight.any() and not d.gate.any()
    assert B.kdkl_last_launch_count() <= 1
