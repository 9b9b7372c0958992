"""The label loss over the C ABI (include/kdkl.h): softmax cross entropy over the LM head against one label a token, beside the
KL loss against a teacher, and like it without the T x V logits.

    ce = LabelLoss(T, H, V, label_smoothing=0.1, z_loss=1e-4)
    loss = ce.forward(hidden, weight, labels)                # [1]; ce.losses and ce.lse [T]
    dhidden, dweight = ce.backward(hidden, weight)           # projects again
    loss, dhidden, dweight = ce.step(hidden, weight, labels) # both at once, three projections for four

The class holds outputs, state and workspaces of one shape: calls only enqueue on the current stream (the first forward call and
the first one that computes gradients also make what they need) and return the holder's own buffers, which the next call
overwrites. Marshalling only; the autograd entry, which allocates its outputs, is ``autograd.label_loss``.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import binding as B
from .body import TYPES, _device, _lookup, _rows, _stream, _vector, _written

REDUCTIONS = {"mean": 0, "sum": 1}
_LABELS = {torch.int32: 0, torch.int64: 1}
_FORWARD, _BACKWARD, _STEP = 0, 1, 2


class kdkl_label_loss_args(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("struct_size", "label_type", "reduction", "dhidden_type", "dweight_type", "accumulate")]
                + [(n, ctypes.c_float) for n in ("temperature", "label_smoothing", "z_loss")] + [("reserved", ctypes.c_int32)]
                + [(n, ctypes.c_int64) for n in ("ignore_index", "T", "H", "V", "chunk")]
                + [(n, ctypes.c_void_p) for n in ("hidden", "weight", "labels", "token_weight", "denom_device", "grad", "grad_tokens", "loss",
                                                  "losses", "lse", "dhidden", "dweight", "state")]
                + [("state_bytes", ctypes.c_size_t), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)])


class LabelLoss:
    """loss = sum over the counted tokens of token_weight * l / D, D their number ("mean") or 1 ("sum"), with
    l = lse - (1 - label_smoothing) z_y - label_smoothing mean(z) + z_loss lse^2, z = hidden @ weight.T / temperature;
    tokens whose label is `ignore_index` are not counted. `dtype` and `dhidden_dtype` are those of the gradients (bf16 or
    fp32). `denom_device`: a CUDA float64 tensor of one element, the divisor in D's place (data-parallel callers)."""

    def __init__(self, T: int, H: int, V: int, *, label_smoothing: float = 0.0, z_loss: float = 0.0, temperature: float = 1.0,
                 ignore_index: int = -100, reduction: str = "mean", chunk: int = 0, dtype=torch.bfloat16, dhidden_dtype=torch.bfloat16,
                 denom_device: Optional[torch.Tensor] = None, train: bool = True, device="cuda"):
        for d in (dtype, dhidden_dtype):
            if d not in (torch.bfloat16, torch.float32):
                raise ValueError(f"kdkl: gradients are bf16 or fp32, not {d}")
        if not 0.0 <= label_smoothing <= 1.0 or not temperature > 0.0:
            raise ValueError(f"kdkl: no label loss with smoothing {label_smoothing} at temperature {temperature}")
        self.T, self.H, self.V, self.train, self.dtype, self.dhidden_dtype = T, H, V, train, dtype, dhidden_dtype
        a = self.args = kdkl_label_loss_args()
        a.struct_size, a.T, a.H, a.V, a.chunk = ctypes.sizeof(a), T, H, V, chunk
        a.reduction, a.ignore_index = _lookup(REDUCTIONS, reduction, "reduction"), ignore_index
        a.temperature, a.label_smoothing, a.z_loss = temperature, label_smoothing, z_loss
        a.dhidden_type, a.dweight_type = TYPES[dhidden_dtype], TYPES[dtype]
        self.denom_device = denom_device
        if denom_device is not None:
            a.denom_device = B._dptr(denom_device, torch.float64, (1,), "denom_device").value
        if not self._need(_FORWARD):
            raise ValueError(f"kdkl: no label loss of shape {(T, H, V)} in chunks of {chunk}")
        a.state_bytes = B.lib().kdkl_label_loss_state_bytes(T)
        self.state = torch.zeros(a.state_bytes, dtype=torch.uint8, device=device)
        self.loss = torch.zeros(1, dtype=torch.float32, device=device)
        self.losses, self.lse = torch.empty(2, T, dtype=torch.float32, device=device).unbind(0)
        a.state, a.loss, a.losses, a.lse = (t.data_ptr() for t in (self.state, self.loss, self.losses, self.lse))
        self.device, self.at = self.state.device, self.state.get_device()
        self.workspaces, self.dhidden, self.dweight, self.token_weight, self.fed = {}, None, None, None, False
        self.gradient_calls = (_BACKWARD, _STEP)                                # those that may come
        self._ref, L = ctypes.byref(a), B.lib()
        self._calls = (L.kdkl_label_loss_forward, L.kdkl_label_loss_backward, L.kdkl_label_loss_step)

    def _need(self, call: int) -> int:
        a = self.args
        return B.lib().kdkl_label_loss_workspace_bytes(a.T, a.H, a.V, a.chunk, call, a.dweight_type)

    def _inputs(self, hidden, weight, labels, token_weight):
        a, T = self.args, self.T
        a.hidden, apart = _rows(hidden, T, self.H, torch.bfloat16, "hidden")
        a.weight, wide = _rows(weight, self.V, self.H, torch.bfloat16, "weight")
        if apart != self.H or wide != self.H:
            raise TypeError("kdkl: hidden and weight: expected contiguous tensors")
        if labels is not None:
            a.label_type = _lookup(_LABELS, labels.dtype, "labels")
            a.labels = _vector(labels, T, labels.dtype, "labels")
        a.token_weight = _vector(token_weight, T, torch.float32, "token_weight")

    def _outputs(self, out, accumulate, want_dhidden=True, want_dweight=True):
        a = self.args
        if not self.train:
            raise RuntimeError("kdkl: this label loss was made for evaluation (train=False)")
        if not (want_dhidden or want_dweight):
            raise ValueError("kdkl: a backward call without a gradient to compute")
        if want_dhidden and self.dhidden is None:
            self.dhidden = torch.empty(self.T, self.H, dtype=self.dhidden_dtype, device=self.device)
        if not want_dweight:
            out = None
        elif out is None:
            if self.dweight is None:
                new = torch.zeros if accumulate else torch.empty                # (a call that does not add writes all of it)
                self.dweight = new(self.V, self.H, dtype=self.dtype, device=self.device)
            out = self.dweight
        else:
            B._dptr(out, self.dtype, (self.V, self.H), "out")
        a.dhidden, a.dweight = self.dhidden.data_ptr() if want_dhidden else None, None if out is None else out.data_ptr()
        a.accumulate = 1 if accumulate else 0
        return (self.dhidden if want_dhidden else None), out

    def _grad(self, grad):
        a = self.args
        a.grad = a.grad_tokens = None
        if grad is None:
            return
        if grad.dim() == 1 and grad.shape[0] == self.T and self.T != 1:
            a.grad_tokens = _vector(grad, self.T, torch.float32, "grad")
        else:
            a.grad = B._dptr(grad.reshape(1) if grad.dim() == 0 else grad, torch.float32, (1,), "grad").value

    def _workspace(self, call: int) -> torch.Tensor:
        """Scratch for a call: backward and step calls share one, which forward calls use where it is there already. None is
        ever replaced, since a captured graph may hold its address."""
        if call == _FORWARD:
            ws = self.workspaces.get("gradients", self.workspaces.get("forward"))
            name, calls = "forward", (_FORWARD,)
        else:
            name, calls = "gradients", self.gradient_calls
            ws = self.workspaces.get(name)
        if ws is None:
            ws = self.workspaces[name] = torch.empty(max(map(self._need, calls)), dtype=torch.uint8, device=self.device)
        return ws

    def _run(self, call: int, written):
        a, ws = self.args, self._workspace(call)
        a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
        B._check(self._calls[call](self._ref, _stream(self.at, "label loss")))
        _written(written)

    def forward(self, hidden, weight, labels, token_weight=None) -> torch.Tensor:
        """The loss [1]; ``losses`` and ``lse`` [T] beside it. Labels are int32 or int64."""
        self._inputs(hidden, weight, labels, token_weight)
        self._run(_FORWARD, [self.loss, self.losses, self.lse, self.state])
        self.token_weight, self.fed = token_weight, True
        return self.loss

    def backward(self, hidden, weight, grad: Optional[torch.Tensor] = None, *, per_token: Optional[bool] = None,
                 out: Optional[torch.Tensor] = None, accumulate: bool = False, want_dhidden: bool = True, want_dweight: bool = True):
        """(dhidden, dweight) after a forward call on the same tensors. `grad`, fp32 on the device: of the loss (one element; 1 if
        None) or of the losses ([T]; `per_token` says which where T is 1). dweight goes to `out` if given; with
        `accumulate` (fp32 only) it is added to what is there. One that is not wanted is None and costs nothing."""
        if not self.fed:
            raise RuntimeError("kdkl: this label loss's backward call comes before any forward call")
        grads = self._outputs(out, accumulate, want_dhidden, want_dweight)
        self._inputs(hidden, weight, None, self.token_weight)
        self._grad(grad)
        if per_token and self.T == 1:
            self.args.grad, self.args.grad_tokens = None, self.args.grad
        self._run(_BACKWARD, [t for t in grads if t is not None])
        return grads

    def step(self, hidden, weight, labels, token_weight=None, grad: Optional[torch.Tensor] = None, *,
             out: Optional[torch.Tensor] = None, accumulate: bool = False, want_dhidden: bool = True, want_dweight: bool = True):
        """(loss, dhidden, dweight) at once, for an upstream gradient of the loss that is known (1 if None)."""
        grads = self._outputs(out, accumulate, want_dhidden, want_dweight)
        self._inputs(hidden, weight, labels, token_weight)
        if grad is not None and grad.numel() != 1:
            raise TypeError(f"kdkl: grad: expected that of the loss, one element, got {tuple(grad.shape)}")
        self.args.grad_tokens, self.args.grad = None, None if grad is None else B._dptr(grad.reshape(1), torch.float32, (1,), "grad").value
        self._run(_STEP, [self.loss, self.losses, self.lse, self.state, *(t for t in grads if t is not None)])
        self.token_weight, self.fed = token_weight, True
        return (self.loss, *grads)

    def status(self):
        """(code, [detail, counted tokens, labels out of range]) of the last calls on this state; waits for them."""
        return B.kdkl_status(self.state)


def rescaled(gradient: torch.Tensor, factor: torch.Tensor) -> torch.Tensor:
    """A gradient that a step has left, times an upstream gradient that became known later (one fp32 element on the device), in a
    tensor of its own: rounded once, and the factor not at all (kdkl_label_loss_rescale)."""
    out = torch.empty_like(gradient)
    B._check(B.lib().kdkl_label_loss_rescale(
        B._dptr(gradient, gradient.dtype, gradient.shape, "gradient"), _lookup(TYPES, gradient.dtype, "gradient"), gradient.numel(),
        B._dptr(factor.reshape(1), torch.float32, (1,), "factor"), out.data_ptr(), _stream(out.get_device(), "gradient")))
    return out
