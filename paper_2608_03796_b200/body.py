"""Operators of a student's body over the C ABI (include/kdkl.h): activations kept in 8 bits and the layers that
read them in the backward pass.

    record = Act8Record(T, H, "int8").store(x)          # x [T, H] -> one byte a value + one per 32
    x_ = record.load()                                  # what it stands for
    dW = Act8WeightGrad(T, N, H).run(dy, record)        # dy^T x_ on the tensor cores, straight from the record
    ffn = GatedAct(T, F); h = ffn.forward(gate, up); dgate, dup = ffn.backward(dh)
    join = BlockNorm(T, H); y, x = join.forward(residual, branch, post_weight=w1, pre_weight=w2)
    d = join.backward(dy, dx)                           # d.residual, d.branch, d.post_weight, d.pre_weight, d.gate

The classes hold outputs, records and workspaces of one shape: calls allocate nothing, only enqueue on the current
stream, and return the holder's own buffers, which the next call overwrites (a graph of autograd's that has saved one of
them raises then). Marshalling only; autograd entries that allocate their outputs are in ``autograd``. Formats are "int8", "e4m3" or None (nothing is kept in 8 bits).
"""
from __future__ import annotations

import ctypes
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
        """The holder's gradient buffer for a weight or gate (made when first needed, or when its type changes)."""
        if like is None:
            return None
        t = self.grads.get(name)
        if t is None or t.dtype != like.dtype:
            t = self.grads[name] = torch.empty_like(like)
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
