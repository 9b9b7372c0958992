"""Operators of a student's body over the C ABI (include/kdkl.h): activations kept in 8 bits and the layers that
read them in the backward pass.

    record = Act8Record(T, H, "int8").store(x)          # x [T, H] -> one byte a value + one per 32
    x_ = record.load()                                  # what it stands for
    dW = Act8WeightGrad(T, N, H).run(dy, record)        # dy^T x_ on the tensor cores, straight from the record
    ffn = GatedAct(T, F); h = ffn.forward(gate, up); dgate, dup = ffn.backward(dh)
    join = BlockNorm(T, H); y, x = join.forward(residual, branch, post_weight=w1, pre_weight=w2)
    d = join.backward(dy, dx)                           # d.residual, d.branch, d.post_weight, d.pre_weight, d.gate
    norm = LayerNorm(T, H); y = norm.forward(x, w, b); d = norm.backward(dy)          # d.x, d.weight, d.bias
    ffn = GatedLinear(T, H, F); h = ffn.forward(x, W_gate_up); dx, dW = ffn.backward(dh)
    rope = Rotary(D); q_, k_ = rope.forward(q, k, positions); dq, dk = rope.backward(dq_, dk_, positions)

The classes hold outputs, records and workspaces of one shape (Rotary: its table, and outputs of the last shape): calls only
enqueue on the current stream and return the holder's own buffers, which the next call overwrites (a graph of autograd's that has
saved one of them raises then). What only a backward pass needs is allocated by the first one, and a Rotary's outputs by
a call of a new shape; calls allocate nothing else. Marshalling only; autograd entries that allocate their outputs are in ``autograd``. Formats are "int8", "e4m3" or None (nothing is kept in 8 bits).
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple, Optional

import torch

from . import binding as B

FORMATS = {None: -1, "int8": 0, "e4m3": 1}
ACTS = {"silu": 0, "gelu": 1}
GATES = {"none": 0, "channel": 1, "token": 2}
TYPES = {torch.bfloat16: 0, torch.float32: 1, torch.float16: 2}
_HALF = (torch.bfloat16, torch.float16)


def _lookup(table, key, name):
    if key not in table:
        raise ValueError(f"kdkl: {name}: expected one of {list(table)}, got {key!r}")
    return table[key]


_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
_capturing = torch._C._cuda_isCurrentStreamCapturing
# The library writes through addresses, which autograd does not see: a graph that has saved a tensor would use the new
# values without a word. Every call therefore says which tensors it has written.
_written = torch.autograd.graph.increment_version


def _rows(t: torch.Tensor, T: int, H: int, dtype, name: str):
    """(address, distance of rows) of a CUDA tensor [T, H] whose rows are contiguous but may lie apart. Refused here,
    as in binding: another device, type or shape, or columns that are not neighbours."""
    at = t.get_device()
    if at < 0 or at != _device() or t.dtype is not dtype or t.shape != (T, H):
        if not t.is_cuda or t.device.index != _device():
            raise TypeError(f"kdkl: {name}: expected a tensor on the current CUDA device, got one on {t.device}")
        if t.dtype != dtype:
            raise TypeError(f"kdkl: {name}: expected dtype {dtype}, got {t.dtype}")
        raise TypeError(f"kdkl: {name}: expected shape {(T, H)}, got {tuple(t.shape)}")
    apart, along = t.stride()
    if (along != 1 and H > 1) or (apart < H and T > 1):
        raise TypeError(f"kdkl: {name}: rows must be contiguous and must not overlap, got strides {t.stride()}")
    return t.data_ptr(), (apart if T > 1 else H)


def _stream(at: int, what: str) -> int:
    """The current stream, for a holder whose own memory is on CUDA device `at` (-1: on the host). The kernels get that
    memory as stored addresses, so a holder from elsewhere is refused here, as binding refuses any such tensor."""
    now = _device()
    if at != now:
        raise TypeError(f"kdkl: {what}: its memory is on {'the host' if at < 0 else f'cuda:{at}'}, but the current device is "
                        f"cuda:{now} (one process per GPU: torch.cuda.set_device first)")
    return _raw_stream(now)


def _vector(t: Optional[torch.Tensor], n: int, dtype, name: str):
    if t is None:
        return None
    at = t.get_device()
    if at >= 0 and at == _device() and t.dtype is dtype and t.shape == (n,) and (n <= 1 or t.stride(0) == 1):
        return t.data_ptr()
    return B._dptr(t, dtype, (n,), name).value                          # says what is wrong


class Act8Record:
    """Activations [T, H] in 8 bits (kdkl_act8_store / kdkl_act8_load). ``buffer`` is the record itself."""

    def __init__(self, T: int, H: int, format: str = "int8", device="cuda", buffer: Optional[torch.Tensor] = None):
        """With `buffer`, the record that it holds already (one of the same shape and format wrote it)."""
        if format is None:
            raise ValueError("kdkl: a record needs a format")
        self.T, self.H, self.format, self.code = T, H, format, _lookup(FORMATS, format, "format")
        self.nbytes = B.lib().kdkl_act8_bytes(T, H)
        if self.nbytes == 0 and T != 0:
            raise ValueError(f"kdkl: no record of shape {(T, H)}")
        if buffer is None:
            buffer = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        elif buffer.dtype != torch.uint8 or not buffer.is_contiguous() or buffer.numel() < self.nbytes:
            raise TypeError(f"kdkl: a record of shape {(T, H)} is {self.nbytes} contiguous bytes")
        self.buffer, self.ptr, self.at = buffer, buffer.data_ptr(), buffer.get_device()
        L = B.lib()
        self._store, self._load = L.kdkl_act8_store, L.kdkl_act8_load

    def store(self, x: torch.Tensor) -> "Act8Record":
        ptr, ld = _rows(x, self.T, self.H, x.dtype, "x")
        B._check(self._store(ptr, _lookup(TYPES, x.dtype, "x"), ld, self.T, self.H, self.code, self.ptr, self.nbytes,
                             _stream(self.at, "record")))
        _written(self.buffer)
        return self

    def load(self, out: Optional[torch.Tensor] = None, dtype=torch.bfloat16) -> torch.Tensor:
        if out is None:
            out = torch.empty(self.T, self.H, dtype=dtype, device=self.buffer.device)
        ptr, ld = _rows(out, self.T, self.H, out.dtype, "out")
        B._check(self._load(self.ptr, self.nbytes, self.T, self.H, self.code, ptr, _lookup(TYPES, out.dtype, "out"), ld,
                            _stream(self.at, "record")))
        _written(out)
        return out


class Act8WeightGrad:
    """dW [N, H] of a linear layer from dy [T, N] (bf16) and the record of its input (kdkl_act8_dweight)."""

    def __init__(self, T: int, N: int, H: int, dtype=torch.bfloat16, device="cuda"):
        if dtype not in (torch.bfloat16, torch.float32):
            raise ValueError(f"kdkl: weight gradients are bf16 or fp32, not {dtype}")
        self.T, self.N, self.H, self.dtype, self.type = T, N, H, dtype, TYPES[dtype]
        nbytes = B.lib().kdkl_act8_dweight_workspace_bytes(T, N, H, self.type)
        if nbytes == 0:
            raise ValueError(f"kdkl: no weight gradient of shape {(T, N, H)}")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.dweight = torch.empty(N, H, dtype=dtype, device=device)
        self.at = self.dweight.get_device()
        self._run, self._own = B.lib().kdkl_act8_dweight, (self.dweight.data_ptr(), self.workspace.data_ptr(), nbytes)

    def run(self, dy: torch.Tensor, record: Act8Record, out: Optional[torch.Tensor] = None,
            accumulate: bool = False) -> torch.Tensor:
        """With `accumulate`, += into `out` (or into the holder's own buffer)."""
        if (record.T, record.H) != (self.T, self.H):
            raise TypeError(f"kdkl: record: expected shape {(self.T, self.H)}, got {(record.T, record.H)}")
        to, workspace, nbytes = self._own
        if out is None:
            out = self.dweight
        else:
            to = B._dptr(out, self.dtype, (self.N, self.H), "out")
        ptr, ld = _rows(dy, self.T, self.N, torch.bfloat16, "dy")
        stream = _stream(record.at, "record")
        B._check(self._run(ptr, ld, record.ptr, record.nbytes, self.T, self.N, self.H, record.code, to, self.type,
                           1 if accumulate else 0, workspace, nbytes,
                           stream if self.at == record.at else _stream(self.at, "weight gradient")))
        _written(out)
        return out

    def status(self):
        """(code, detail) of the last run, which waits for it; every run starts with a clear status."""
        return B.kdkl_status(self.workspace)


class GatedAct:
    """h = act(gate) * up (kdkl_gated_act_forward / _backward). With act8 given the forward call leaves records of gate
    and up, which the backward call reads; with keep_h also one of h (``h_record``, for the layer that reads h)."""

    def __init__(self, T: int, F: int, act: str = "silu", act8: Optional[str] = "int8", dtype=torch.bfloat16,
                 keep_h: bool = False, device="cuda"):
        if dtype not in _HALF:
            raise ValueError(f"kdkl: gated activations are bf16 or fp16, not {dtype}")
        self.T, self.F, self.dtype, self.type = T, F, dtype, TYPES[dtype]
        self.act, self.format = _lookup(ACTS, act, "act"), _lookup(FORMATS, act8, "act8")
        self.h = torch.empty(T, F, dtype=dtype, device=device)
        self.device, self.at, self._h = self.h.device, self.h.get_device(), self.h.data_ptr()
        self._forward, self._backward = B.lib().kdkl_gated_act_forward, B.lib().kdkl_gated_act_backward
        self.gate_record = self.up_record = self.h_record = None
        self.dgate_up, self.stored = None, False
        if act8 is not None:
            self.gate_record, self.up_record = Act8Record(T, F, act8, device), Act8Record(T, F, act8, device)
            self.h_record = Act8Record(T, F, act8, device) if keep_h else None

    def forward(self, gate: torch.Tensor, up: torch.Tensor) -> torch.Tensor:
        g, ld = _rows(gate, self.T, self.F, self.dtype, "gate")
        u, ld_u = _rows(up, self.T, self.F, self.dtype, "up")
        if ld_u != ld:
            raise TypeError(f"kdkl: gate and up must have their rows equally far apart, got {ld} and {ld_u}")
        keep, also, written = self.gate_record, self.h_record, [self.h]
        records = (None, None, None, 0)
        if keep is not None:
            records = (keep.ptr, self.up_record.ptr, None if also is None else also.ptr, keep.nbytes)
            written += [keep.buffer, self.up_record.buffer] if also is None else [keep.buffer, self.up_record.buffer, also.buffer]
        B._check(self._forward(g, u, ld, self.type, self.T, self.F, self.act, self.format, self._h, self.F, *records,
                               _stream(self.at, "gated activation")))
        _written(written)
        self.stored = True
        return self.h

    def backward(self, dh: torch.Tensor):
        """(dgate, dup), the halves of one [T, 2 F] buffer."""
        if self.gate_record is None:
            raise RuntimeError("kdkl: this gated activation keeps nothing for a backward pass (act8=None)")
        if not self.stored:
            raise RuntimeError("kdkl: this gated activation's backward call comes before any forward call")
        if self.dgate_up is None:
            self.dgate_up = torch.empty(self.T, 2 * self.F, dtype=self.dtype, device=self.device)
            self.halves = self.dgate_up[:, :self.F], self.dgate_up[:, self.F:]
        d, ld = _rows(dh, self.T, self.F, self.dtype, "dh")
        for kept in (self.gate_record, self.up_record):
            if kept.at != self.at:                                          # (autograd's hooks may have moved it)
                _stream(kept.at, "record")
        out = self.dgate_up.data_ptr()
        B._check(self._backward(
            self.gate_record.ptr, self.up_record.ptr, self.gate_record.nbytes, self.format, d, ld, self.type, self.T, self.F, self.act,
            out, out + self.F * self.dtype.itemsize, 2 * self.F, _stream(self.at, "gated activation")))
        _written(self.dgate_up)
        return self.halves


class BlockNormGrads(NamedTuple):
    residual: torch.Tensor
    branch: torch.Tensor
    post_weight: Optional[torch.Tensor]
    pre_weight: Optional[torch.Tensor]
    gate: Optional[torch.Tensor]


class kdkl_block_norm_args(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("struct_size", "type", "residual_type", "weight_type", "gate_type",
                                               "gate_kind", "format")]
                + [(n, ctypes.c_float) for n in ("eps", "weight_offset", "branch_scale", "residual_scale")]
                + [("T", ctypes.c_int64), ("H", ctypes.c_int64), ("residual", ctypes.c_void_p),
                   ("ld_residual", ctypes.c_int64), ("branch", ctypes.c_void_p), ("ld_branch", ctypes.c_int64)]
                + [(n, ctypes.c_void_p) for n in ("post_weight", "pre_weight", "gate", "y", "sum", "rho_post", "rho_pre",
                                                  "branch_record", "sum_record", "y_record")]
                + [("record_bytes", ctypes.c_size_t), ("dy", ctypes.c_void_p), ("ld_dy", ctypes.c_int64),
                   ("dsum", ctypes.c_void_p), ("ld_dsum", ctypes.c_int64)]
                + [(n, ctypes.c_void_p) for n in ("dresidual", "dbranch", "dpost_weight", "dpre_weight", "dgate",
                                                  "workspace")]
                + [("workspace_bytes", ctypes.c_size_t)])


class BlockNorm:
    """The join between two blocks (kdkl_block_norm_forward / _backward):

        n = branch * rsqrt(mean(branch^2) + eps) * (post_weight + weight_offset)     (post_weight None: n = branch)
        x = residual_scale * residual + branch_scale * gate * n
        y = x * rsqrt(mean(x^2) + eps) * (pre_weight + weight_offset)                (pre_weight None: y is None)

    `gate` is "none", "channel" ([H]) or "token" ([T]). With act8 given, forward leaves records of branch and x, which
    backward reads; otherwise backward reads the tensors, which the caller leaves in place. keep_y: a record of y too
    (``y_record``, for the layer that reads y). train=False keeps nothing."""

    def __init__(self, T: int, H: int, *, dtype=torch.bfloat16, residual_dtype=None, gate: str = "none",
                 act8: Optional[str] = None, eps: float = 1e-6, weight_offset: float = 0.0, branch_scale: float = 1.0,
                 residual_scale: float = 1.0, train: bool = True, keep_y: bool = False, device="cuda"):
        residual_dtype = residual_dtype or dtype
        if dtype not in _HALF or residual_dtype not in (dtype, torch.float32):
            raise ValueError(f"kdkl: a block norm is bf16 or fp16, its residual the same or fp32, not {dtype}, {residual_dtype}")
        self.T, self.H, self.dtype, self.residual_dtype, self.train = T, H, dtype, residual_dtype, train
        a = self.args = kdkl_block_norm_args()
        a.struct_size = ctypes.sizeof(a)
        a.type, a.residual_type, a.weight_type, a.gate_type = TYPES[dtype], TYPES[residual_dtype], 0, 0
        a.gate_kind = _lookup(GATES, gate, "gate")
        keeps = train and act8 is not None
        a.format = _lookup(FORMATS, act8, "act8") if keeps else -1
        a.eps, a.weight_offset, a.branch_scale, a.residual_scale = eps, weight_offset, branch_scale, residual_scale
        a.T, a.H = T, H
        self.y = torch.empty(T, H, dtype=dtype, device=device)
        self.sum = torch.empty(T, H, dtype=residual_dtype, device=device)
        a.y, a.sum, self.at = self.y.data_ptr(), self.sum.data_ptr(), self.y.get_device()
        self.branch_record = self.sum_record = self.y_record = None
        self.workspace = self.dresidual = self.dbranch = None               # made by the first backward call
        if train:
            self.workspace_bytes = B.lib().kdkl_block_norm_workspace_bytes(T, H)
            if self.workspace_bytes == 0:
                raise ValueError(f"kdkl: no block norm of shape {(T, H)}")
            self.rho = torch.empty(2, T, dtype=torch.float32, device=device)
            a.rho_post, a.rho_pre = self.rho[0].data_ptr(), self.rho[1].data_ptr()
        if keeps:
            self.branch_record, self.sum_record = Act8Record(T, H, act8, device), Act8Record(T, H, act8, device)
            self.y_record = Act8Record(T, H, act8, device) if keep_y else None
        self.grads, self.kept = {}, None
        self._ref = ctypes.byref(a)
        self._forward, self._backward = B.lib().kdkl_block_norm_forward, B.lib().kdkl_block_norm_backward

    def forward(self, residual, branch, post_weight=None, pre_weight=None, gate=None):
        """(y, x); y is None without a pre_weight."""
        if pre_weight is None and self.y_record is not None:
            raise ValueError("kdkl: keep_y needs a pre_weight: without one there is no y, and its record would stay another call's")
        a = self.args
        a.residual, a.ld_residual = _rows(residual, self.T, self.H, self.residual_dtype, "residual")
        a.branch, a.ld_branch = _rows(branch, self.T, self.H, self.dtype, "branch")
        self._weights(post_weight, pre_weight, gate)
        written = self._records()
        written += (self.sum,) if pre_weight is None else (self.sum, self.y)
        B._check(self._forward(self._ref, _stream(self.at, "block norm")))
        _written(written)
        if self.train:                                                      # what the backward call reads
            self.kept = (*((branch, self.sum) if a.format < 0 else (None, None)), post_weight, pre_weight, gate)
        return (self.y if pre_weight is not None else None), self.sum

    def _weights(self, post_weight, pre_weight, gate):
        a, H = self.args, self.H
        w = post_weight if post_weight is not None else pre_weight
        if w is not None:
            a.weight_type = _lookup(TYPES, w.dtype, "norm weight")
            a.post_weight = _vector(post_weight, H, w.dtype, "post_weight")
            a.pre_weight = _vector(pre_weight, H, w.dtype, "pre_weight")
        else:
            a.post_weight = a.pre_weight = None
        if (gate is None) != (a.gate_kind == 0):
            raise TypeError(f"kdkl: gate: given {gate is not None}, but this block norm was made with gate kind {a.gate_kind}")
        if gate is not None:
            a.gate_type = _lookup(TYPES, gate.dtype, "gate")
            a.gate = _vector(gate, H if a.gate_kind == 1 else self.T, gate.dtype, "gate")

    def _records(self):
        """Their memory goes into the arguments and is returned."""
        a, buffers = self.args, []
        if a.format >= 0:
            for kept in (self.branch_record, self.sum_record, self.y_record):
                if kept is not None:
                    if kept.at != self.at:                                  # (autograd's hooks may have moved it)
                        _stream(kept.at, "record")
                    buffers.append(kept.buffer)
            a.branch_record, a.sum_record = self.branch_record.ptr, self.sum_record.ptr
            a.y_record = None if self.y_record is None else self.y_record.ptr
            a.record_bytes = self.branch_record.nbytes
        return buffers

    def _grad(self, name, like):
        """The holder's gradient buffer for a weight or gate (made when first needed, one for each type: the kernels of another
        stream may still be at work on what would be given up)."""
        if like is None:
            return None
        t = self.grads.get((name, like.dtype))
        if t is None:
            t = self.grads[name, like.dtype] = torch.empty_like(like)
        return t

    def backward(self, dy, dsum=None) -> BlockNormGrads:
        """Gradients of the last forward call's inputs from those of y (None without a pre norm) and of x."""
        if not self.train:
            raise RuntimeError("kdkl: this block norm keeps nothing for a backward pass (train=False)")
        if self.kept is None:
            raise RuntimeError("kdkl: this block norm's backward call comes before any forward call")
        a = self.args
        if self.workspace is None:
            device = self.rho.device
            self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device)
            self.dresidual = torch.empty(self.T, self.H, dtype=self.residual_dtype, device=device)
            self.dbranch = torch.empty(self.T, self.H, dtype=self.dtype, device=device)
            a.workspace, a.workspace_bytes = self.workspace.data_ptr(), self.workspace_bytes
            a.dresidual, a.dbranch = self.dresidual.data_ptr(), self.dbranch.data_ptr()
        branch, total, post_weight, pre_weight, gate = self.kept
        self._weights(post_weight, pre_weight, gate)
        self._records()
        if a.format < 0:
            a.branch, a.ld_branch = _rows(branch, self.T, self.H, self.dtype, "branch")
            a.sum = _rows(total, self.T, self.H, self.residual_dtype, "sum")[0]
        if (dy is None) != (pre_weight is None):
            raise TypeError("kdkl: dy goes with a pre_weight")
        if dy is not None:
            a.dy, a.ld_dy = _rows(dy, self.T, self.H, self.dtype, "dy")
        if dsum is not None:
            a.dsum, a.ld_dsum = _rows(dsum, self.T, self.H, self.residual_dtype, "dsum")
        else:
            a.dsum = None
        d = BlockNormGrads(self.dresidual, self.dbranch, self._grad("post", post_weight), self._grad("pre", pre_weight),
                           self._grad("gate", gate))
        a.dpost_weight = None if d.post_weight is None else d.post_weight.data_ptr()
        a.dpre_weight = None if d.pre_weight is None else d.pre_weight.data_ptr()
        a.dgate = None if d.gate is None else d.gate.data_ptr()
        B._check(self._backward(self._ref, _stream(self.at, "block norm")))
        _written([t for t in d if t is not None])
        return d


class kdkl_layer_norm_args(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("struct_size", "x_type", "y_type", "weight_type", "format")]
                + [("eps", ctypes.c_float), ("T", ctypes.c_int64), ("H", ctypes.c_int64), ("x", ctypes.c_void_p), ("ld_x", ctypes.c_int64)]
                + [(n, ctypes.c_void_p) for n in ("weight", "bias", "y", "mean", "rho", "x_record", "y_record")]
                + [("record_bytes", ctypes.c_size_t), ("dy", ctypes.c_void_p), ("ld_dy", ctypes.c_int64)]
                + [(n, ctypes.c_void_p) for n in ("dx", "dweight", "dbias", "workspace")] + [("workspace_bytes", ctypes.c_size_t)])


class LayerNormGrads(NamedTuple):
    x: torch.Tensor
    weight: Optional[torch.Tensor]
    bias: Optional[torch.Tensor]


class LayerNorm:
    """y = (x - mean(x)) * rsqrt(var(x) + eps) * weight + bias per row of x [T, H] (kdkl_layer_norm_forward / _backward);
    weight None: ones, bias None: zeros. `dtype` is that of y and dy, `x_dtype` of x and dx (dtype's own, or fp32). With
    act8 given, forward leaves a record of x, which backward reads; otherwise backward reads the tensor, which the caller
    leaves in place. keep_y: a record of y too (``y_record``, for the layer that reads y). train=False keeps nothing."""

    def __init__(self, T: int, H: int, *, dtype=torch.bfloat16, x_dtype=None, act8: Optional[str] = None, eps: float = 1e-5,
                 train: bool = True, keep_y: bool = False, device="cuda"):
        x_dtype = x_dtype or dtype
        if dtype not in TYPES or x_dtype not in (dtype, torch.float32):
            raise ValueError(f"kdkl: a layer norm is bf16, fp16 or fp32, its input the same or fp32, not {dtype}, {x_dtype}")
        if keep_y and not (train and act8 is not None):
            raise ValueError("kdkl: keep_y needs act8, in training")
        self.T, self.H, self.dtype, self.x_dtype, self.train = T, H, dtype, x_dtype, train
        a = self.args = kdkl_layer_norm_args()
        a.struct_size = ctypes.sizeof(a)
        a.x_type, a.y_type, a.weight_type = TYPES[x_dtype], TYPES[dtype], 0
        a.format = _lookup(FORMATS, act8, "act8") if train else -1
        a.eps, a.T, a.H = eps, T, H
        self.y = torch.empty(T, H, dtype=dtype, device=device)
        a.y, self.at = self.y.data_ptr(), self.y.get_device()
        self.x_record = self.y_record = self.workspace = self.dx = self.kept = None
        if train:
            self.workspace_bytes = B.lib().kdkl_layer_norm_workspace_bytes(T, H)
            if self.workspace_bytes == 0:
                raise ValueError(f"kdkl: no layer norm of shape {(T, H)}")
            self.stats = torch.empty(2, T, dtype=torch.float32, device=device)
            a.mean, a.rho = self.stats[0].data_ptr(), self.stats[1].data_ptr()
            if act8 is not None:
                self.x_record = Act8Record(T, H, act8, device)
                self.y_record = Act8Record(T, H, act8, device) if keep_y else None
        self.grads = {}
        self._ref = ctypes.byref(a)
        self._forward, self._backward = B.lib().kdkl_layer_norm_forward, B.lib().kdkl_layer_norm_backward

    def forward(self, x, weight=None, bias=None) -> torch.Tensor:
        a = self.args
        a.x, a.ld_x = _rows(x, self.T, self.H, self.x_dtype, "x")
        self._affine(weight, bias)
        written = self._records()
        B._check(self._forward(self._ref, _stream(self.at, "layer norm")))
        _written([self.y, *written])
        if self.train:                                                      # what the backward call reads
            self.kept = (x if a.format < 0 else None, weight, bias)
        return self.y

    def _affine(self, weight, bias):
        a, given = self.args, weight if weight is not None else bias
        if given is None:
            a.weight = a.bias = None
            return
        a.weight_type = _lookup(TYPES, given.dtype, "weight")
        a.weight, a.bias = _vector(weight, self.H, given.dtype, "weight"), _vector(bias, self.H, given.dtype, "bias")

    def _records(self):
        a, kept = self.args, [r for r in (self.x_record, self.y_record) if r is not None]
        for r in kept:
            if r.at != self.at:                                             # (autograd's hooks may have moved it)
                _stream(r.at, "record")
            a.record_bytes = r.nbytes
        a.x_record = None if self.x_record is None else self.x_record.ptr
        a.y_record = None if self.y_record is None else self.y_record.ptr
        return [r.buffer for r in kept]

    def _grad(self, name, like):
        """As BlockNorm's."""
        if like is None:
            return None
        t = self.grads.get((name, like.dtype))
        if t is None:
            t = self.grads[name, like.dtype] = torch.empty_like(like)
        return t

    def backward(self, dy) -> LayerNormGrads:
        """Gradients of the last forward call's inputs."""
        if not self.train:
            raise RuntimeError("kdkl: this layer norm keeps nothing for a backward pass (train=False)")
        if self.kept is None:
            raise RuntimeError("kdkl: this layer norm's backward call comes before any forward call")
        a = self.args
        if self.workspace is None:
            self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=self.stats.device)
            a.workspace, a.workspace_bytes = self.workspace.data_ptr(), self.workspace_bytes
        if self.dx is None:
            self.dx = torch.empty(self.T, self.H, dtype=self.x_dtype, device=self.stats.device)
            a.dx = self.dx.data_ptr()
        x, weight, bias = self.kept
        self._affine(weight, bias)
        self._records()
        if a.format < 0:
            a.x, a.ld_x = _rows(x, self.T, self.H, self.x_dtype, "x")
        a.dy, a.ld_dy = _rows(dy, self.T, self.H, self.dtype, "dy")
        d = LayerNormGrads(self.dx, self._grad("weight", weight), self._grad("bias", bias))
        a.dweight = None if d.weight is None else d.weight.data_ptr()
        a.dbias = None if d.bias is None else d.bias.data_ptr()
        B._check(self._backward(self._ref, _stream(self.at, "layer norm")))
        _written([t for t in d if t is not None])
        return d


LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}
_POSITIONS = {torch.int32: 0, torch.int64: 1}


class kdkl_rotary_args(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("struct_size", "type", "layout", "head_dim", "rotary_dim", "q_heads", "k_heads",
                                               "wide_positions", "inverse")]
                + [("magnitude", ctypes.c_float), ("T", ctypes.c_int64), ("positions", ctypes.c_void_p), ("turns", ctypes.c_void_p)]
                + [f for n in ("q", "q_out", "k", "k_out")
                   for f in ((n, ctypes.c_void_p), (n + "_token", ctypes.c_int64), (n + "_head", ctypes.c_int64))])


class Rotary:
    """Rotary positions of queries [T, heads, D] and keys [T, kv heads, D] (kdkl_rotary). The first `rotary_dim` columns of a
    head (all by default) are pairs - "half": (i, i + rotary_dim / 2), "interleaved": (2 i, 2 i + 1) - turned by
    position * base ** (-2 i / rotary_dim) radians. `scaling` ("linear", "ntk", "yarn", by `factor`) is for contexts longer
    than `original_length`, the one that was trained on; see kdkl_rotary_table for the formulas. "yarn" is that of its paper: how
    much of a frequency is kept is linear in its turns over the trained length, none at 1 and all at 32. Much model code takes
    it linear in the pair's index between the places of those two, which turns the middle pairs by other angles: a
    checkpoint wants the ones that it was trained with. Those, or any others, are given as `frequencies`, rotary_dim / 2 numbers
    of radians a position in place of base and scaling; `magnitude` is the factor on turned columns, in place of scaling's.

    Tokens and heads may lie any distance apart (the halves of one projection, or x.transpose(0, 1) of heads before
    tokens); columns are neighbours. Outputs are the holder's own buffers, made for each stream and new shape, or those given as
    `out` (which may be the inputs themselves: then they are changed in place). A call that is captured into a graph makes new
    ones, which live in the graph's memory and belong to the caller. Threads that share a table give their outputs, or each has
    a stream of its own."""

    def __init__(self, D: int, rotary_dim: Optional[int] = None, *, base: float = 10000.0, layout: str = "half",
                 scaling: str = "none", factor: float = 1.0, original_length: int = 0, frequencies=None,
                 magnitude: Optional[float] = None, device="cuda"):
        R = D if rotary_dim is None else rotary_dim
        if D % 2 or R % 2 or not 2 <= R <= D <= 1024:
            raise ValueError(f"kdkl: heads of {D} columns, {R} of them turned: both are even, and at most 1024")
        a = self.args = kdkl_rotary_args()
        kind = _lookup(SCALINGS, scaling, "scaling")
        if frequencies is None:
            turns, m = (ctypes.c_double * (R // 2))(), ctypes.c_float()
            if B.lib().kdkl_rotary_table(R, base, kind, factor, original_length, turns, ctypes.byref(m)) != 0:
                raise ValueError(f"kdkl: no rotary positions with base {base}, scaling {scaling!r} by {factor} of {original_length}")
            turns, m = torch.tensor(list(turns), dtype=torch.float64), m.value
        else:
            turns, m = torch.as_tensor(frequencies, dtype=torch.float64).cpu() / (2 * math.pi), 1.0
            if kind != 0 or turns.shape != (R // 2,) or not torch.isfinite(turns).all():
                raise ValueError(f"kdkl: frequencies: expected {R // 2} finite numbers, without a scaling, got shape "
                                 f"{tuple(turns.shape)}, scaling {scaling!r}")
        m = m if magnitude is None else float(magnitude)
        if not math.isfinite(m):
            raise ValueError(f"kdkl: magnitude: expected a finite number, got {magnitude}")
        self.D, self.R = D, R
        a.struct_size = ctypes.sizeof(a)
        a.layout, a.head_dim, a.rotary_dim, a.magnitude = _lookup(LAYOUTS, layout, "layout"), D, R, m
        self.turns = turns.to(device)
        a.turns, self.at = self.turns.data_ptr(), self.turns.get_device()
        self._call, self._streams, self._own = B.lib().kdkl_rotary, {}, {}

    def forward(self, q, k, positions, out=None):
        """(q, k) turned; k may be None."""
        return self._run(q, k, positions, out, 0)

    def backward(self, dq, dk, positions, out=None):
        """Gradients of q and k from those of their turned forms."""
        return self._run(dq, dk, positions, out, 1)

    def _run(self, q, k, positions, out, inverse):
        a = kdkl_rotary_args.from_buffer_copy(self.args)     # a call's own: threads that give outputs may share a table
        now, dtype, D, T = _device(), q.dtype, self.D, positions.shape[0] if positions.dim() == 1 else -1
        if positions.get_device() != now or positions.dtype not in _POSITIONS or T < 0 or (T > 1 and positions.stride(0) != 1):
            raise TypeError(f"kdkl: positions: expected contiguous int32 or int64 [T] on the current CUDA device, got "
                            f"{positions.dtype} {tuple(positions.shape)} on {positions.device}")
        a.T, a.positions, a.wide_positions, a.inverse, a.type = T, positions.data_ptr(), _POSITIONS[positions.dtype], inverse, \
            _lookup(TYPES, dtype, "q")
        heads, a.q, a.q_token, a.q_head = self._heads(q, T, dtype, "q", now)
        a.q_heads, stream = heads, _stream(self.at, "rotary table")
        if out is None:
            captured = _capturing()
            own = self._buffers(stream)
            y = self._buffer(own, inverse, 0, q, captured)
            a.q_out, a.q_out_token, a.q_out_head = y.data_ptr(), heads * D, D
        else:
            y = out[0]
            n, a.q_out, a.q_out_token, a.q_out_head = self._heads(y, T, dtype, "q's output", now)
            self._same(n, heads)
        if k is None:
            a.k_heads, outs, written = 0, (y, None), y
        else:
            heads, a.k, a.k_token, a.k_head = self._heads(k, T, dtype, "k", now)
            a.k_heads = heads
            if out is None:
                z = self._buffer(own, inverse, 1, k, captured)
                a.k_out, a.k_out_token, a.k_out_head = z.data_ptr(), heads * D, D
            else:
                z = out[1]
                n, a.k_out, a.k_out_token, a.k_out_head = self._heads(z, T, dtype, "k's output", now)
                self._same(n, heads)
            outs = written = (y, z)
        B._check(self._call(ctypes.byref(a), stream))
        _written(written)
        return outs

    @staticmethod
    def _same(given, heads):
        if given != heads:
            raise TypeError(f"kdkl: an output of {given} heads for an input of {heads}")

    def _heads(self, t, T, dtype, name, now):
        """(heads, address, distance of tokens, distance of heads)"""
        if t.dim() == 3:
            (n, heads, wide), (token, head, along) = t.shape, t.stride()
            if n == T and wide == self.D and along == 1 and t.dtype is dtype and t.get_device() == now:
                return heads, t.data_ptr(), token, head
        raise TypeError(f"kdkl: {name}: expected {dtype} [{T}, heads, {self.D}] on the current CUDA device, columns contiguous, "
                        f"got {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")

    def _buffers(self, stream):
        """The outputs of calls on a stream. The allocator gives what is dropped to later work of the stream that it was made
        on: a buffer that calls on two streams write could not be replaced while the other one's are under way."""
        own = self._streams.get(stream)
        if own is None:
            own = self._streams.setdefault(stream, {})
        self._own = own
        return own

    def _buffer(self, own, inverse, which, like, captured):
        if captured:                        # the graph's memory, the caller's to keep: a replay must not write into eager calls' outputs
            return torch.empty(like.shape, dtype=like.dtype, device=like.device)
        t = own.get((inverse, which))
        if t is None or t.shape != like.shape or t.dtype is not like.dtype or t.device != like.device:
            t = own[inverse, which] = torch.empty(like.shape, dtype=like.dtype, device=like.device)
        return t


class kdkl_gated_linear_args(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("struct_size", "act", "format", "dweight_type", "accumulate", "reserved")]
                + [(n, ctypes.c_int64) for n in ("T", "H", "F")]
                + [("x", ctypes.c_void_p), ("ld_x", ctypes.c_int64), ("weight", ctypes.c_void_p), ("h", ctypes.c_void_p),
                   ("ld_h", ctypes.c_int64)]
                + [(n, ctypes.c_void_p) for n in ("gate_record", "up_record", "h_record")]
                + [("record_bytes", ctypes.c_size_t), ("x_record", ctypes.c_void_p), ("x_record_bytes", ctypes.c_size_t),
                   ("dh", ctypes.c_void_p), ("ld_dh", ctypes.c_int64)]
                + [(n, ctypes.c_void_p) for n in ("dgate_up", "dx", "dweight", "workspace")] + [("workspace_bytes", ctypes.c_size_t)])


class GatedLinear:
    """h = act(x @ Wg.T) * (x @ Wu.T) of x [T, H] and the stacked weight [2 F, H] (Wg above Wu), in one kernel
    (kdkl_gated_linear_forward / _backward). bf16; H and F are multiples of 8.

    With act8 given, forward leaves records of gate and up, which backward reads, together with a record of x that
    whoever made x left; keep_h: a record of h too (``h_record``, for the layer that reads h). With act8=None nothing
    is kept beside x itself, which the caller leaves in place, and backward forms gate and up again. train=False: no
    backward call. `dtype` is that of the weight's gradient (bf16 or fp32)."""

    def __init__(self, T: int, H: int, F: int, *, act: str = "silu", act8: Optional[str] = None, train: bool = True,
                 keep_h: bool = False, dtype=torch.bfloat16, device="cuda"):
        if dtype not in (torch.bfloat16, torch.float32):
            raise ValueError(f"kdkl: weight gradients are bf16 or fp32, not {dtype}")
        if keep_h and not (train and act8 is not None):
            raise ValueError("kdkl: keep_h needs act8, in training")
        self.T, self.H, self.F, self.dtype, self.train, self.act8 = T, H, F, dtype, train, act8
        a = self.args = kdkl_gated_linear_args()
        a.struct_size, a.T, a.H, a.F = ctypes.sizeof(a), T, H, F
        a.act, a.format, a.dweight_type = _lookup(ACTS, act, "act"), _lookup(FORMATS, act8, "act8") if train else -1, TYPES[dtype]
        self.workspace_bytes = B.lib().kdkl_gated_linear_workspace_bytes(T, H, F, a.dweight_type)
        if self.workspace_bytes == 0:
            raise ValueError(f"kdkl: no gated linear layer of shape {(T, H, F)}")
        self.h = torch.empty(T, F, dtype=torch.bfloat16, device=device)
        self.head = torch.zeros(256, dtype=torch.uint8, device=device)          # the forward call's status
        self.device, self.at = self.h.device, self.h.get_device()
        a.h, a.ld_h = self.h.data_ptr(), F
        self.gate_record = self.up_record = self.h_record = self.kept = None
        if a.format >= 0:
            self.gate_record, self.up_record = Act8Record(T, F, act8, device), Act8Record(T, F, act8, device)
            self.h_record = Act8Record(T, F, act8, device) if keep_h else None
        self.workspace = self.dgate_up = self.dx = self.dweight = None          # made by the first backward call
        self._ref, self.last = ctypes.byref(a), self.head
        self._forward, self._backward = B.lib().kdkl_gated_linear_forward, B.lib().kdkl_gated_linear_backward

    def forward(self, x: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
        a = self.args
        a.x, a.ld_x = _rows(x, self.T, self.H, torch.bfloat16, "x")
        self._weight(weight)
        written = self._records()
        a.workspace, a.workspace_bytes = self.head.data_ptr(), 256
        B._check(self._forward(self._ref, _stream(self.at, "gated linear layer")))
        _written([self.h, *written])
        self.last = self.head
        if self.train:                                                      # what the backward call reads
            self.kept = (x if a.format < 0 else None, weight)
        return self.h

    def _weight(self, weight):
        ptr, apart = _rows(weight, 2 * self.F, self.H, torch.bfloat16, "weight")
        if apart != self.H:
            raise TypeError(f"kdkl: weight: expected a contiguous tensor, got strides {weight.stride()}")
        self.args.weight = ptr

    def _records(self):
        a, kept = self.args, [r for r in (self.gate_record, self.up_record, self.h_record) if r is not None]
        for r in kept:
            if r.at != self.at:                                             # (autograd's hooks may have moved it)
                _stream(r.at, "record")
            a.record_bytes = r.nbytes
        a.gate_record, a.up_record, a.h_record = (None if r is None else r.ptr for r in (self.gate_record, self.up_record, self.h_record))
        return [r.buffer for r in kept]

    def backward(self, dh: torch.Tensor, record: Optional[Act8Record] = None, *, out: Optional[torch.Tensor] = None,
                 accumulate: bool = False, want_dx: bool = True, want_dweight: bool = True):
        """(dx, dweight) of the last forward call's inputs. `record` is that of x, needed with act8 for the weight's gradient,
        which goes to `out` if given; with `accumulate` it is added to what is there."""
        if not self.train:
            raise RuntimeError("kdkl: this gated linear layer keeps nothing for a backward pass (train=False)")
        if self.kept is None:
            raise RuntimeError("kdkl: this gated linear layer's backward call comes before any forward call")
        a, bf16 = self.args, torch.bfloat16
        if want_dweight and a.format >= 0:
            if record is None or (record.T, record.H, record.code) != (self.T, self.H, a.format):
                raise TypeError(f"kdkl: record: expected one of x, {(self.T, self.H)} {self.act8}, got "
                                f"{None if record is None else (record.T, record.H, record.format)}")
            if record.at != self.at:
                _stream(record.at, "record")
            a.x_record, a.x_record_bytes = record.ptr, record.nbytes
        if self.workspace is None:
            self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=self.device)
        if self.dgate_up is None:
            self.dgate_up = torch.empty(self.T, 2 * self.F, dtype=bf16, device=self.device)
        if want_dx and self.dx is None:
            self.dx = torch.empty(self.T, self.H, dtype=bf16, device=self.device)
        if not want_dweight:
            out = None
        elif out is not None:
            B._dptr(out, self.dtype, (2 * self.F, self.H), "out")
        else:
            if self.dweight is None:
                self.dweight = torch.empty(2 * self.F, self.H, dtype=self.dtype, device=self.device)
            out = self.dweight
        x, weight = self.kept
        self._weight(weight)
        self._records()
        if a.format < 0:
            a.x, a.ld_x = _rows(x, self.T, self.H, bf16, "x")
        a.dh, a.ld_dh = _rows(dh, self.T, self.F, bf16, "dh")
        a.dgate_up, a.dx = self.dgate_up.data_ptr(), self.dx.data_ptr() if want_dx else None
        a.dweight, a.accumulate = None if out is None else out.data_ptr(), 1 if accumulate else 0
        a.workspace, a.workspace_bytes = self.workspace.data_ptr(), self.workspace_bytes
        B._check(self._backward(self._ref, _stream(self.at, "gated linear layer")))
        _written([t for t in (self.dgate_up, self.dx if want_dx else None, out) if t is not None])
        self.last = self.workspace
        return (self.dx if want_dx else None), out

    def status(self):
        """(code, detail) of the last call, which waits for it; every call starts with a clear status."""
        return B.kdkl_status(self.last)
