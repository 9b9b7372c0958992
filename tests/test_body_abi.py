"""Argument checks of the student-body operators: found on the host before any CUDA call, so checked without a GPU.
Pointers are made up but not null and aligned: nothing dereferences them on these paths."""
import ctypes

import pytest
import torch

import __graft_entry__ as entry
from paper_2608_03796_b200 import binding as B
from paper_2608_03796_b200 import body

NULL, SHAPE, ALIGN, SPACE, ARG = -1, -2, -3, -4, -5
P, Q, R = 0x100000, 0x200000, 0x300000
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    entry.build()
    return B.lib()


def test_record_sizes(L):
    for T, H in [(1, 1), (1, 4096), (333, 2816), (5, 33), (1 << 20, 4096)]:
        Hp = (H + 31) // 32 * 32
        Sp = (Hp // 32 + 15) // 16 * 16
        need = (T * Hp + 255) // 256 * 256 + T * Sp
        got = L.kdkl_act8_bytes(T, H)
        assert need <= got < need + 256 and got % 256 == 0
    assert L.kdkl_act8_bytes(1 << 20, 8192) > 1 << 32                   # offsets past 32 bits
    assert L.kdkl_act8_bytes(0, 64) == 0 and L.kdkl_act8_bytes(-1, 64) == 0 and L.kdkl_act8_bytes(4, 0) == 0


def test_record_refusals(L):
    def store(x=P, type=0, ld=64, T=4, H=64, fmt=0, rec=Q, nbytes=BIG):
        return L.kdkl_act8_store(x, type, ld, T, H, fmt, rec, nbytes, None)

    def load(out=P, type=0, ld=64, T=4, H=64, fmt=0, rec=Q, nbytes=BIG):
        return L.kdkl_act8_load(rec, nbytes, T, H, fmt, out, type, ld, None)
    for f, x in ((store, "x"), (load, "out")):
        assert f(**{x: None}) == NULL and f(rec=None) == NULL
        assert f(T=-1) == SHAPE and f(H=0) == SHAPE and f(ld=63) == SHAPE
        assert f(type=3) == ARG and f(type=-1) == ARG and f(fmt=-1) == ARG and f(fmt=2) == ARG
        assert f(rec=Q + 16) == ALIGN and f(**{x: P + 1}) == ALIGN and f(type=1, **{x: P + 2}) == ALIGN
        assert f(nbytes=4 * 64) == SPACE
        assert f(T=0) == 0 and f(T=0, **{x: None}) == 0


def test_gated_refusals(L):
    def fwd(g=P, u=P, ld=64, type=0, T=4, F=64, act=0, fmt=0, h=P, ld_h=64, rg=Q, ru=R, rh=None, nbytes=BIG):
        return L.kdkl_gated_act_forward(g, u, ld, type, T, F, act, fmt, h, ld_h, rg, ru, rh, nbytes, None)

    def bwd(rg=Q, ru=R, nbytes=BIG, fmt=0, dh=P, ld_dh=64, type=0, T=4, F=64, act=0, dg=P, du=P, ld=128):
        return L.kdkl_gated_act_backward(rg, ru, nbytes, fmt, dh, ld_dh, type, T, F, act, dg, du, ld, None)
    assert fwd(g=None) == NULL and fwd(u=None) == NULL and fwd(h=None) == NULL
    assert fwd(rg=None) == NULL and fwd(ru=None) == NULL
    assert fwd(type=1) == ARG and fwd(act=2) == ARG and fwd(fmt=2) == ARG and fwd(fmt=-2) == ARG
    assert fwd(F=0) == SHAPE and fwd(ld=63) == SHAPE and fwd(ld_h=1) == SHAPE and fwd(T=-3) == SHAPE
    assert fwd(rg=Q + 1) == ALIGN and fwd(rh=Q + 16) == ALIGN and fwd(g=P + 1) == ALIGN
    assert fwd(nbytes=10) == SPACE and fwd(T=0) == 0
    assert bwd(rg=None) == NULL and bwd(dh=None) == NULL and bwd(dg=None) == NULL and bwd(du=None) == NULL
    assert bwd(fmt=-1) == ARG and bwd(type=1) == ARG and bwd(act=-1) == ARG
    assert bwd(ld=32) == SHAPE and bwd(ld_dh=32) == SHAPE and bwd(nbytes=3) == SPACE and bwd(ru=R + 8) == ALIGN


def test_dweight_refusals(L):
    ws = L.kdkl_act8_dweight_workspace_bytes(4, 32, 64, 0)
    assert ws > 0 and L.kdkl_act8_dweight_workspace_bytes(4, 32, 64, 2) == 0

    def dw(dy=P, ld=32, rec=Q, nbytes=BIG, T=4, N=32, H=64, fmt=0, out=P, type=0, acc=0, w=R, wb=ws):
        return L.kdkl_act8_dweight(dy, ld, rec, nbytes, T, N, H, fmt, out, type, acc, w, wb, None)
    assert dw(dy=None) == NULL and dw(rec=None) == NULL and dw(out=None) == NULL and dw(w=None) == NULL
    assert dw(N=0) == SHAPE and dw(H=0) == SHAPE and dw(ld=31) == SHAPE and dw(T=-1) == SHAPE
    assert dw(type=2) == ARG and dw(acc=2) == ARG and dw(fmt=3) == ARG
    assert dw(w=R + 8) == ALIGN and dw(dy=P + 1) == ALIGN and dw(out=P + 2, type=1) == ALIGN
    assert dw(wb=ws - 1) == SPACE and dw(nbytes=7) == SPACE


def test_norm_refusals(L):
    def args(**kw):
        a = body.kdkl_block_norm_args()
        a.struct_size = ctypes.sizeof(a)
        a.format, a.eps, a.branch_scale, a.residual_scale, a.T, a.H = -1, 1e-6, 1.0, 1.0, 4, 64
        for n in ("residual", "branch", "post_weight", "pre_weight", "y", "sum", "rho_post", "rho_pre", "dy", "dsum",
                  "dresidual", "dbranch", "dpost_weight", "dpre_weight", "workspace"):
            setattr(a, n, P)
        a.ld_residual = a.ld_branch = a.ld_dy = a.ld_dsum = 64
        a.workspace_bytes = BIG
        for k, v in kw.items():
            setattr(a, k, v)
        return a
    fwd = lambda **kw: L.kdkl_block_norm_forward(ctypes.byref(args(**kw)), None)       # noqa: E731
    bwd = lambda **kw: L.kdkl_block_norm_backward(ctypes.byref(args(**kw)), None)      # noqa: E731
    assert L.kdkl_block_norm_forward(None, None) == NULL
    for f in (fwd, bwd):
        assert f(struct_size=8) == ARG and f(type=1) == ARG and f(residual_type=2) == ARG and f(weight_type=5) == ARG
        assert f(gate_kind=3) == ARG and f(format=2) == ARG and f(eps=-1.0) == ARG and f(eps=float("nan")) == ARG
        assert f(branch_scale=float("inf")) == ARG
        assert f(gate_kind=1) == NULL and f(gate_kind=2) == NULL
        assert f(H=0) == SHAPE and f(H=32769) == SHAPE and f(T=-1) == SHAPE and f(ld_branch=63) == SHAPE
        assert f(post_weight=P + 1) == ALIGN and f(rho_post=P + 2) == ALIGN
        assert f(format=0, branch_record=Q + 16, record_bytes=BIG) == ALIGN
        assert f(format=0, branch_record=Q, record_bytes=5) == SPACE
    assert fwd(residual=None) == NULL and fwd(branch=None) == NULL and fwd(sum=None) == NULL and fwd(y=None) == NULL
    assert fwd(ld_residual=1) == SHAPE and fwd(branch=P + 1) == ALIGN and fwd(T=0) == 0
    for n in ("dresidual", "dbranch", "dpost_weight", "dpre_weight", "dy", "rho_post", "rho_pre", "workspace", "branch", "sum"):
        assert bwd(**{n: None}) == NULL, n
    assert bwd(format=1, sum_record=Q, record_bytes=BIG) == NULL and bwd(format=1, branch_record=Q, record_bytes=BIG) == NULL
    assert bwd(ld_dy=3) == SHAPE and bwd(ld_dsum=3) == SHAPE
    assert bwd(workspace=P + 8) == ALIGN and bwd(workspace_bytes=16) == SPACE and bwd(dy=P + 1) == ALIGN
    assert L.kdkl_block_norm_workspace_bytes(4, 40000) == 0


def test_python_refusals_without_a_gpu(L):
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        body.Act8Record(4, 64, "int4", device="cpu")
    with pytest.raises(ValueError):
        body.Act8Record(4, 64, None, device="cpu")
    with pytest.raises(TypeError):
        body.Act8Record(4, 64, device="cpu").store(x)                   # a host tensor
    with pytest.raises(TypeError):
        body.GatedAct(4, 64, device="cpu").forward(x, x)
    with pytest.raises(ValueError):
        body.GatedAct(4, 64, dtype=torch.float32, device="cpu")
    with pytest.raises(ValueError):
        body.GatedAct(4, 64, act="relu", device="cpu")
    with pytest.raises(ValueError):
        body.Act8WeightGrad(4, 8, 8, dtype=torch.float16, device="cpu")
    with pytest.raises(ValueError):
        body.BlockNorm(4, 64, residual_dtype=torch.float16, device="cpu")
    with pytest.raises(ValueError):
        body.BlockNorm(4, 64, gate="head", device="cpu")
    with pytest.raises(ValueError):
        body.BlockNorm(4, 40000, device="cpu")


def test_args_struct_is_the_headers(L, tmp_path):
    """sizeof and every field's offset, as a C compiler sees them."""
    import os
    import shutil
    import subprocess
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no gcc")
    names = [n for n, _ in body.kdkl_block_norm_args._fields_]
    src = tmp_path / "offsets.c"
    src.write_text('#include <stdio.h>\n#include "kdkl.h"\nint main(void) { printf("%zu\\n", sizeof(kdkl_block_norm_args));\n'
                   + "".join(f'printf("%zu\\n", offsetof(kdkl_block_norm_args, {n}));\n' for n in names) + "return 0; }\n")
    exe = tmp_path / "offsets"
    subprocess.run([gcc, "-std=c99", "-I", os.path.join(entry.ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got[0] == ctypes.sizeof(body.kdkl_block_norm_args)
    assert got[1:] == [getattr(body.kdkl_block_norm_args, n).offset for n in names]
