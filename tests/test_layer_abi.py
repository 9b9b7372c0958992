"""Argument checks of the layer norm and of rotary positions: found on the host before any CUDA call, so checked without a
GPU (pointers are made up but not null and aligned); and the rotary table, which is host arithmetic."""
import ctypes
import math
import re

import pytest
import torch

from paper_2608_03796_b200 import binding as B
from paper_2608_03796_b200 import body
from tests.test_body_sources import _code

NULL, SHAPE, ALIGN, SPACE, ARG = -1, -2, -3, -4, -5
P, Q = 0x100000, 0x200000
BIG = 1 << 40


def _norm(backward=False, **kw):
    a = body.kdkl_layer_norm_args()
    fields = dict(struct_size=ctypes.sizeof(a), x_type=0, y_type=0, weight_type=0, format=-1, eps=1e-5, T=4, H=64, x=P, ld_x=64,
                  weight=P, bias=P, y=P, mean=P, rho=P, x_record=Q, y_record=None, record_bytes=BIG, dy=P, ld_dy=64, dx=P,
                  dweight=P, dbias=P, workspace=Q, workspace_bytes=BIG)
    fields.update(kw)
    for k, v in fields.items():
        setattr(a, k, v)
    f = B.lib().kdkl_layer_norm_backward if backward else B.lib().kdkl_layer_norm_forward
    return f(ctypes.byref(a), None)


def test_layer_norm_refusals():
    for back in (False, True):
        assert _norm(back, struct_size=8) == ARG and _norm(back, T=-1) == SHAPE and _norm(back, H=0) == SHAPE
        assert _norm(back, x_type=3) == ARG and _norm(back, weight_type=-1) == ARG
        assert _norm(back, x_type=0, y_type=2) == ARG and _norm(back, x_type=2, y_type=1) == ARG
        assert _norm(back, format=2) == ARG and _norm(back, format=-2) == ARG
        assert _norm(back, eps=-1.0) == ARG and _norm(back, eps=math.nan) == ARG and _norm(back, eps=math.inf) == ARG
        assert _norm(back, weight=P + 1) == ALIGN and _norm(back, bias=P + 2, weight_type=1) == ALIGN
        assert _norm(back, ld_x=63) == SHAPE and _norm(back, x=None) == NULL and _norm(back, x=P + 1) == ALIGN
        assert _norm(back, format=0, record_bytes=100) == SPACE and _norm(back, format=0, x_record=Q + 16) == ALIGN
    assert _norm(y=None) == NULL and _norm(mean=None) == NULL and _norm(rho=None) == NULL and _norm(y=P + 1) == ALIGN
    assert _norm(T=0, x=None, y=None) == 0
    for name in ("dy", "dx", "dweight", "dbias", "workspace", "mean", "rho"):
        assert _norm(True, **{name: None}) == NULL, name
    assert _norm(True, format=1, x_record=None) == NULL
    assert _norm(True, ld_dy=10) == SHAPE and _norm(True, workspace=Q + 64) == ALIGN and _norm(True, workspace_bytes=255) == SPACE
    assert B.lib().kdkl_layer_norm_forward(None, None) == NULL and B.lib().kdkl_layer_norm_backward(None, None) == NULL
    assert B.lib().kdkl_layer_norm_workspace_bytes(-1, 64) == 0 and B.lib().kdkl_layer_norm_workspace_bytes(4, 0) == 0
    assert B.lib().kdkl_layer_norm_workspace_bytes(0, 64) > 0


def _rotary(**kw):
    a = body.kdkl_rotary_args()
    fields = dict(struct_size=ctypes.sizeof(a), type=0, layout=0, head_dim=64, rotary_dim=64, q_heads=4, k_heads=2, wide_positions=1,
                  inverse=0, magnitude=1.0, T=8, positions=P, turns=P, q=P, q_token=256, q_head=64, q_out=Q, q_out_token=256,
                  q_out_head=64, k=P, k_token=128, k_head=64, k_out=Q, k_out_token=128, k_out_head=64)
    fields.update(kw)
    for k, v in fields.items():
        setattr(a, k, v)
    return B.lib().kdkl_rotary(ctypes.byref(a), None)


def test_rotary_refusals():
    assert B.lib().kdkl_rotary(None, None) == NULL and _rotary(struct_size=4) == ARG
    for bad in (dict(T=-1), dict(head_dim=63), dict(head_dim=0), dict(head_dim=2048), dict(rotary_dim=66), dict(rotary_dim=31),
                dict(rotary_dim=0), dict(q_heads=-1), dict(k_heads=5000), dict(q_token=-1), dict(k_head=-64)):
        assert _rotary(**bad) == SHAPE, bad
    # outputs whose heads or tokens would overlap
    for bad in (dict(q_out_head=63), dict(q_out_token=63), dict(q_out_token=128), dict(k_out_head=64, k_out_token=64)):
        assert _rotary(**bad) == SHAPE, bad
    for bad in (dict(type=3), dict(layout=2), dict(inverse=2), dict(wide_positions=2), dict(magnitude=math.inf)):
        assert _rotary(**bad) == ARG, bad
    for name in ("positions", "turns", "q", "q_out", "k", "k_out"):
        assert _rotary(**{name: None}) == NULL, name
    assert _rotary(positions=P + 4) == ALIGN and _rotary(turns=P + 4) == ALIGN and _rotary(q=P + 1) == ALIGN
    assert _rotary(type=1, k_out=Q + 2) == ALIGN
    assert _rotary(T=0, q=None) == 0 and _rotary(q_heads=0, k_heads=0) == 0


def _table(R, base=10000.0, scaling=0, factor=1.0, length=0.0):
    turns, m = (ctypes.c_double * max(1, R // 2))(), ctypes.c_float()
    rc = B.lib().kdkl_rotary_table(R, base, scaling, factor, length, turns, ctypes.byref(m))
    return rc, list(turns), m.value


@pytest.mark.parametrize("scaling", [0, 1, 2, 3])
def test_rotary_table(scaling):
    R, base, s, L = 64, 50000.0, 8.0, 4096.0
    rc, turns, m = _table(R, base, scaling, s, L)
    assert rc == 0
    for i, got in enumerate(turns):
        b = base * s ** (R / (R - 2)) if scaling == 2 else base
        f = b ** (-2 * i / R)
        if scaling == 1:
            f /= s
        if scaling == 3:
            k = min(1.0, max(0.0, (L * f / (2 * math.pi) - 1) / 31))
            f = k * f + (1 - k) * f / s
        assert abs(got * 2 * math.pi - f) <= 1e-14 * f
    assert m == pytest.approx(1 + 0.1 * math.log(s) if scaling == 3 else 1.0, rel=1e-7)
    if scaling == 3:                                                        # the fastest pair is kept, the slowest is stretched
        assert turns[0] == pytest.approx(1 / (2 * math.pi)) and turns[-1] * 2 * math.pi == pytest.approx(base ** (-62 / 64) / s)


def test_rotary_table_refusals():
    assert _table(0)[0] == SHAPE and _table(3)[0] == SHAPE and _table(2048)[0] == SHAPE and _table(2, scaling=2, factor=2.0)[0] == SHAPE
    assert _table(8, base=1.0)[0] == ARG and _table(8, base=math.nan)[0] == ARG and _table(8, scaling=4)[0] == ARG
    assert _table(8, scaling=1, factor=0.5)[0] == ARG and _table(8, scaling=1, factor=math.inf)[0] == ARG
    assert _table(8, scaling=3, factor=2.0, length=0.0)[0] == ARG
    assert B.lib().kdkl_rotary_table(8, 1e4, 0, 1.0, 0.0, None, None) == NULL


def test_holders_refuse():
    with pytest.raises(ValueError):
        body.Rotary(63, device="cpu")
    with pytest.raises(ValueError):
        body.Rotary(64, rotary_dim=66, device="cpu")
    with pytest.raises(ValueError):
        body.Rotary(64, scaling="cubic", device="cpu")
    with pytest.raises(ValueError):
        body.Rotary(64, scaling="yarn", factor=2.0, device="cpu")           # of which length?
    with pytest.raises(ValueError):
        body.LayerNorm(4, 64, dtype=torch.float64, device="cpu")
    with pytest.raises(ValueError):
        body.LayerNorm(4, 64, x_dtype=torch.float16, device="cpu")
    with pytest.raises(ValueError):
        body.LayerNorm(4, 64, keep_y=True, device="cpu")
    with pytest.raises(ValueError):
        body.LayerNorm(4, 0, device="cpu")
    with pytest.raises(RuntimeError, match="before any forward"):
        body.LayerNorm(4, 64, device="cpu").backward(torch.zeros(4, 64))
    with pytest.raises(RuntimeError, match="keeps nothing"):
        body.LayerNorm(4, 64, train=False, device="cpu").backward(torch.zeros(4, 64))


def test_memory_on_the_host_is_refused_before_a_launch(monkeypatch):
    monkeypatch.setattr(body, "_rows", lambda t, T, H, dtype, name: (P, H))
    monkeypatch.setattr(body, "_vector", lambda t, n, dtype, name: P)
    monkeypatch.setattr(body, "_device", lambda: 0)
    monkeypatch.setattr(body, "_raw_stream", lambda device: 0)

    def reached(*args):
        raise AssertionError("an address of another device reached the library")
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.ones(64, dtype=torch.bfloat16)
    norm = body.LayerNorm(4, 64, device="cpu")
    norm._forward = norm._backward = reached
    norm.kept = (x, w, w)
    for call in (lambda: norm.forward(x, w, w), lambda: norm.backward(x)):
        with pytest.raises(TypeError, match="on the host"):
            call()
    rope = body.Rotary(64, device="cpu")
    rope._call = reached
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        rope.forward(q, q, torch.arange(4))


@pytest.mark.parametrize("name", ["layer_norm_kernels.cuh", "rotary_kernels.cuh"])
def test_kernels_that_start_early_read_coherently(name):
    code = _code(name)
    assert "grid_dependency_wait" in code and "__restrict__" not in code
    assert not re.search(r"\.nc\b", code) and "__ldg" not in code


def _gated(backward=False, **kw):
    a = body.kdkl_gated_linear_args()
    fields = dict(struct_size=ctypes.sizeof(a), act=0, format=-1, dweight_type=0, accumulate=0, T=16, H=64, F=64, x=P, ld_x=64, weight=P,
                  h=P, ld_h=64, gate_record=Q, up_record=Q, h_record=None, record_bytes=BIG, x_record=Q, x_record_bytes=BIG, dh=P,
                  ld_dh=64, dgate_up=P, dx=P, dweight=P, workspace=Q, workspace_bytes=BIG)
    fields.update(kw)
    for k, v in fields.items():
        setattr(a, k, v)
    f = B.lib().kdkl_gated_linear_backward if backward else B.lib().kdkl_gated_linear_forward
    return f(ctypes.byref(a), None)


def test_gated_linear_refusals():
    for back in (False, True):
        assert _gated(back, struct_size=1) == ARG and _gated(back, act=2) == ARG and _gated(back, format=2) == ARG
        for bad in (dict(T=-1), dict(H=0), dict(H=60), dict(F=4), dict(F=0), dict(F=1 << 29), dict(ld_x=56)):
            assert _gated(back, **bad) == SHAPE, bad
        assert _gated(back, weight=None) == NULL and _gated(back, workspace=None) == NULL and _gated(back, x=None) == NULL
        assert _gated(back, weight=P + 2) == ALIGN and _gated(back, workspace=Q + 16) == ALIGN and _gated(back, x=P + 8) == ALIGN
        assert _gated(back, ld_x=68) == ALIGN and _gated(back, workspace_bytes=255) == SPACE
        assert _gated(back, format=0, gate_record=None) == NULL and _gated(back, format=1, up_record=None) == NULL
        assert _gated(back, format=0, record_bytes=64) == SPACE and _gated(back, format=0, up_record=Q + 16) == ALIGN
    assert _gated(h=None) == NULL and _gated(ld_h=63) == SHAPE and _gated(h=P + 8) == ALIGN and _gated(T=0, x=None, h=None) == 0
    assert _gated(format=0, h_record=Q + 32) == ALIGN
    assert _gated(True, dh=None) == NULL and _gated(True, dgate_up=None) == NULL and _gated(True, format=0, x_record=None) == NULL
    assert _gated(True, dweight_type=2) == ARG and _gated(True, accumulate=2) == ARG
    assert _gated(True, ld_dh=32) == SHAPE and _gated(True, dx=P + 4) == ALIGN and _gated(True, dweight=P + 4) == ALIGN
    assert _gated(True, format=0, x_record_bytes=8) == SPACE
    size = B.lib().kdkl_gated_linear_workspace_bytes
    assert size(16, 60, 64, 0) == 0 and size(16, 64, 64, 2) == 0 and size(-1, 64, 64, 0) == 0 and size(0, 64, 64, 1) >= 256
    with pytest.raises(ValueError):
        body.GatedLinear(4, 60, 64, device="cpu")
    with pytest.raises(ValueError):
        body.GatedLinear(4, 64, 64, dtype=torch.float16, device="cpu")
    with pytest.raises(ValueError):
        body.GatedLinear(4, 64, 64, keep_h=True, device="cpu")
    with pytest.raises(RuntimeError, match="keeps nothing"):
        body.GatedLinear(4, 64, 64, train=False, device="cpu").backward(torch.zeros(4, 64))
