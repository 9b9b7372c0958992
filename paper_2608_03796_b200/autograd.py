"""torch.autograd entry to the fused chunked KL loss (and the optional feature loss).

    loss = fused_chunked_kl(hidden, weight, topk_idx, topk_val, teacher_lse=None, loss_mask=None,
                            chunk=4096, temperature=1.0)
    loss.backward()          # hidden.grad [T,H] bf16, weight.grad [V,H] bf16 (rounded from the fp32 dW)

Marshalling only: forward runs kdkl_forward, backward runs kdkl_backward; nothing of the loss arithmetic
happens in torch ops. Neither call waits for the device: the upstream gradient stays where autograd holds it
(kdkl_options.grad_loss_device), and the device status of a step (a bounded wait that ran out, a state mismatch)
is copied to pinned host memory behind the step's kernels and looked at when the same buffers are next used, or
by check_status() - an error of step i is therefore raised during step i+1. `sync_status=True` reads the status
at the end of backward instead (one stream synchronisation per step). The single-pass form compares the upstream
gradient with `expected_grad` on the host and so reads it once (`grad.item()`).
Workspace and gradient buffers are pooled per shape, so repeated steps allocate nothing. A forward call takes a
buffer set out of the pool and owns it until its backward has run: two losses of one shape that are both alive
(loss1 + loss2, pipelined micro-batches, activation checkpointing) therefore never share the saved state of
Algorithm 1, and a backward whose buffer set has been reused in the meantime (a second backward through a freed
graph) raises instead of returning gradients of another batch. `weight_grad_fp32=True` hands the fp32 dW
buffer over to the caller (the pool allocates a new one next time) instead of a bf16 copy; with `dweight_out`
given, dW is accumulated into that fp32 tensor in place.

    loss = label_loss(hidden, weight, labels, label_smoothing=0.1)     # hard labels; reduction "mean", "sum" or "none"

is the same for one label a token (``labels``): only a few numbers a token live between its two passes, workspaces come from
torch's allocator for the length of a call.

The layers of a student's body whose backward pass reads activations kept in 8 bits (``body``):

    y, x, kept = block_norm(x, branch, post_weight, pre_weight, gate, act8="int8", keep_y=True)
    z = act8_linear(y, W_gate_up, record=kept)               # keeps nothing of its own
    h, kept = gated_act(z, act="silu", act8="int8", keep_h=True)
    branch = act8_linear(h, W_down, record=kept)
    y, kept = layer_norm(x, weight, bias, act8="int8", keep_y=True)
    q, k = rotary(q, k, positions, body.Rotary(D))
    h, kept = gated_linear(y, W_gate_up, act8="int8", record=kept, keep_h=True)     # act8_linear and gated_act in one kernel

Their outputs, records and gradients are allocated per call, as a graph needs them.
"""
from __future__ import annotations

import functools
from typing import Optional

import torch

from . import binding as B
from . import body
from . import labels as L


class _NoSecondDerivative(torch.autograd.Function):
    @staticmethod
    def forward(ctx, name, anchor, *grads):
        ctx.name = name
        return tuple(g.view_as(g) for g in grads)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError(f"{ctx.name}: the backward pass is computed by kernels that have no derivative, so there are no "
                           "second derivatives through it")


def _first_derivative_only(name):
    """For the backward pass of a Function whose kernels autograd cannot differentiate. Under create_graph its gradients
    come back as ever, but a graph that depends on them raises when it is differentiated: their dependence on the saved
    tensors would otherwise be missing in silence (whether or not the upstream gradient needs a graph itself)."""
    def wrap(backward):
        @functools.wraps(backward)
        def once(ctx, *grads):
            if not torch.is_grad_enabled():
                return backward(ctx, *grads)
            with torch.no_grad():
                out = backward(ctx, *grads)
            outs = list(out if isinstance(out, tuple) else (out,))
            at = [i for i, t in enumerate(outs) if isinstance(t, torch.Tensor)]
            if at:
                for i, t in zip(at, _NoSecondDerivative.apply(name, torch.empty(0, requires_grad=True), *(outs[i] for i in at))):
                    outs[i] = t
            return tuple(outs)
        return once
    return wrap


_free: dict = {}          # key -> buffer sets (FusedChunkedKL holders) no live loss is using
_probed: list = []        # buffer sets whose last step's status has not been looked at yet
_idle: list = []          # _StepStatus objects that wait for nothing
_captured: list = []      # (what, status words) of steps that a CUDA graph repeats


def clear_cache() -> None:
    """Drops the pooled workspaces and gradient buffers (sets in use by a live loss are unaffected)."""
    try:
        check_status()
    finally:
        _free.clear()
        _captured.clear()


def _probe(op) -> None:
    """Enqueue a copy of the workspace header's status words to pinned host memory behind the step's kernels."""
    if getattr(op, "probe", None) is None:
        op.probe = torch.zeros(4, dtype=torch.int32).pin_memory()
        op.probe_event = torch.cuda.Event()
    op.probe.copy_(op.workspace[:16].view(torch.int32), non_blocking=True)
    op.probe_event.record()
    if not getattr(op, "probe_pending", False):
        op.probe_pending = True
        _probed.append(op)


def _collect(op) -> None:
    """Look at the status a finished earlier step left (waits for that step's kernels only if they still run)."""
    if not getattr(op, "probe_pending", False):
        return
    op.probe_event.synchronize()
    op.probe_pending = False
    if op in _probed:
        _probed.remove(op)
    code, where = int(op.probe[0]), int(op.probe[1])
    if code not in (0, -10):                                      # -10: out-of-range teacher indices were ignored
        what = getattr(op, "what", "fused_chunked_kl")
        if isinstance(op, _StepStatus):
            _idle.append(op)
        raise B.KdklError(code, f"device status of an earlier {what} step, detail {where}")
    if isinstance(op, _StepStatus):
        _idle.append(op)


class _StepStatus:
    """The status of one step whose workspace is not kept: 16 bytes of pinned memory and an event."""
    what = ""


def _watch(workspace, what: str) -> None:
    """Remembers the status words that the step just enqueued leaves in `workspace` for check_status, and looks at those
    of earlier such steps that have ended."""
    if torch.cuda.is_current_stream_capturing():
        words = torch.empty(4, dtype=torch.int32, device=workspace.device)     # every replay writes them again
        words.copy_(workspace[:16].view(torch.int32))
        _captured.append((what, words))
        return
    op = _idle.pop() if _idle else _StepStatus()
    op.what, op.workspace = what, workspace
    _probe(op)
    op.workspace = None
    for earlier in [q for q in _probed if isinstance(q, _StepStatus) and q is not op]:
        if not earlier.probe_event.query():
            break                                             # (in the order of the steps)
        _collect(earlier)


def check_status() -> None:
    """Raises if any step whose status has not been looked at yet failed on the device (waits for those steps), or the last
    replay of a step that a CUDA graph repeats."""
    first = None
    for op in list(_probed):                   # every pending status is collected, the first failure is raised
        try:
            _collect(op)
        except B.KdklError as e:
            first = first or e
    for what, words in _captured:
        code, where = words[:2].tolist()
        if code == -8:                         # KDKL_ERR_TIMEOUT (before the first replay the words are anything)
            first = first or B.KdklError(code, f"device status of a captured {what} step, detail {where}")
    if first is not None:
        raise first


def _acquire(T, H, V, K, chunk, tau, accumulate, device):
    """A buffer set for this shape that nothing else is using: out of the pool, or a new one."""
    key = (T, H, V, K, chunk, tau, accumulate, str(device))
    pool = _free.setdefault(key, [])
    if pool:
        op = pool.pop()
        _collect(op)                                              # the status its last step left
        if op.dweight is None:                                    # handed over to a caller last time
            op.dweight = torch.empty(V, H, dtype=torch.float32, device=device)
    else:
        op = B.FusedChunkedKL(T, H, V, K, chunk=chunk, temperature=tau,
                              opt=B.make_options(accumulate_dweight=accumulate), device=device)
        op.generation = 0
    op.generation += 1
    return key, op


def _release(key, op) -> None:
    _free.setdefault(key, []).append(op)


class _FusedChunkedKL(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, topk_idx, topk_val, teacher_lse, loss_mask, chunk, temperature, dweight_out,
                weight_grad_fp32, single_pass, expected_grad, sync_status):
        T, H = hidden.shape
        V, K = weight.shape[0], topk_idx.shape[1]
        # single pass: the gradients for an upstream gradient of 1 come out of the forward call (three projections
        # instead of four); it writes dW itself, so it is not combined with accumulation into a caller's buffer
        ctx.done = bool(single_pass) and dweight_out is None
        key, op = _acquire(T, H, V, K, int(chunk), float(temperature), 1 if dweight_out is not None else 0,
                           hidden.device)
        ctx.expected = float(expected_grad)
        if ctx.done:
            op.forward_backward(hidden, weight, topk_idx, topk_val, teacher_lse=teacher_lse, loss_mask=loss_mask,
                                grad_loss=ctx.expected)
        else:
            op.forward(hidden, weight, topk_idx, topk_val, teacher_lse=teacher_lse, loss_mask=loss_mask)
        loss = op.loss.clone().squeeze(0)
        if not (ctx.needs_input_grad[0] or ctx.needs_input_grad[1]):
            _release(key, op)                                     # no backward will come: the set is free again
            return loss
        ctx.op, ctx.key, ctx.generation, ctx.mask = op, key, op.generation, loss_mask
        ctx.dweight_out, ctx.weight_grad_fp32, ctx.sync_status = dweight_out, weight_grad_fp32, bool(sync_status)
        ctx.save_for_backward(hidden, weight)
        return loss

    @staticmethod
    @_first_derivative_only("fused_chunked_kl")
    def backward(ctx, grad):
        hidden, weight = ctx.saved_tensors
        op = ctx.op
        if op.generation != ctx.generation:
            raise RuntimeError("fused_chunked_kl: this loss's saved state has been reused by a later forward call "
                               "(backward ran twice without retain_graph semantics the buffers can honour)")
        if not (ctx.done and float(grad.item()) == ctx.expected):   # any other upstream gradient: the recompute path
            if ctx.dweight_out is not None:
                saved, op.dweight = op.dweight, ctx.dweight_out   # dW += into the caller's fp32 buffer
            try:                                                  # the upstream gradient stays on the device
                op.backward(hidden, weight, loss_mask=ctx.mask,
                            grad_loss=grad.detach().to(torch.float32).contiguous())
            finally:
                if ctx.dweight_out is not None:
                    op.dweight = saved
        if ctx.sync_status:
            code, detail = op.status()
            if code not in (0, -10):                              # -10: out-of-range teacher indices were ignored
                raise B.KdklError(code, f"device status, detail {detail}")
        else:
            _probe(op)
        if ctx.dweight_out is not None:
            dW = None
        elif ctx.weight_grad_fp32:
            dW, op.dweight = op.dweight, None                     # ownership passes to the caller
        else:
            dW = op.dweight.to(weight.dtype)
        dH = op.dhidden.clone()
        _release(ctx.key, op)          # free for the next forward; a second backward of this graph before that
        return dH, dW, None, None, None, None, None, None, None, None, None, None, None   # still finds its state intact


def fused_chunked_kl(hidden, weight, topk_idx, topk_val, teacher_lse: Optional[torch.Tensor] = None,
                     loss_mask: Optional[torch.Tensor] = None, chunk: int = 4096, temperature: float = 1.0,
                     dweight_out: Optional[torch.Tensor] = None, weight_grad_fp32: bool = False,
                     single_pass: bool = False, expected_grad: float = 1.0, sync_status: bool = False) -> torch.Tensor:
    """Mean forward KL between the cached top-K teacher and softmax(hidden @ weight.T / temperature).
    single_pass=True computes the gradients during the forward call (kdkl_forward_backward) for an upstream
    gradient of `expected_grad` (the weight this loss carries in the total); if backward then sees another
    value, the gradients are recomputed by kdkl_backward."""
    return _FusedChunkedKL.apply(hidden, weight, topk_idx, topk_val, teacher_lse, loss_mask, chunk, temperature,
                                 dweight_out, weight_grad_fp32, single_pass, expected_grad, sync_status)


class _FeatureLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, student, teacher, loss_mask, kind, weight):
        T, H = student.shape
        ws = torch.empty(B.kdkl_feature_loss_workspace_bytes(T), dtype=torch.uint8, device=student.device)
        loss = torch.zeros(1, dtype=torch.float32, device=student.device)
        B.kdkl_feature_loss(student, teacher, ws, loss, kind=kind, loss_mask=loss_mask, weight=weight)   # loss only
        ctx.save_for_backward(student, teacher, ws)
        ctx.args = (loss_mask, kind, weight)
        return loss.squeeze(0)

    @staticmethod
    @_first_derivative_only("feature_loss")
    def backward(ctx, g):
        # one more pass of the same kernel writes grad * d loss / d student; the upstream gradient stays on the device
        student, teacher, ws = ctx.saved_tensors
        loss_mask, kind, weight = ctx.args
        grad = torch.empty_like(student)
        scratch = torch.zeros(1, dtype=torch.float32, device=student.device)
        B.kdkl_feature_loss(student, teacher, ws, scratch, kind=kind, loss_mask=loss_mask, weight=weight,
                            grad_loss=g.detach().to(torch.float32).contiguous(), dstudent=grad)
        return grad, None, None, None, None


def feature_loss(student, teacher, loss_mask=None, kind=B.FEATURE_MSE, weight=1.0) -> torch.Tensor:
    """Hidden-state feature loss (MSE or cosine) between student and cached teacher hidden states."""
    return _FeatureLoss.apply(student, teacher, loss_mask, kind, weight)


def _flat(t: torch.Tensor, width: int) -> torch.Tensor:
    """[..., width] as rows whose columns are neighbours and which do not overlap (a copy where they do)."""
    t = t.reshape(-1, width)
    apart, along = t.stride()
    return t if (along == 1 or width == 1) and (apart >= width or t.shape[0] <= 1) else t.contiguous()


def _shaped(t: torch.Tensor, shape) -> torch.Tensor:
    """The memory of a contiguous tensor under another shape, not as a view of it: what a Function returns may then be
    changed in place like any other tensor."""
    return t if t.shape == shape else torch.empty(0, dtype=t.dtype, device=t.device).set_(t.untyped_storage(), 0, shape)


def _recorded(*tensors) -> bool:
    """Whether a backward pass can come (within a Function's forward, grad mode is off and does not say)."""
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


class _Act8Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, record, act8, keep, sync_status):
        N, H = weight.shape
        rows = _flat(x, H)
        if keep:
            if record is None:
                record = body.Act8Record(rows.shape[0], H, act8, device=x.device).store(rows)
            elif (record.T, record.H) != tuple(rows.shape):
                raise TypeError(f"act8_linear: the record is of shape {(record.T, record.H)}, the input of {tuple(rows.shape)}")
            ctx.format, ctx.sync_status = record.format, sync_status
        ctx.save_for_backward(weight, None if record is None else record.buffer)
        ctx.shape = x.shape
        return torch.matmul(rows, weight.t()).reshape(*x.shape[:-1], N)          # a plain library product

    @staticmethod
    @_first_derivative_only("act8_linear")
    def backward(ctx, dy):
        weight, buffer = ctx.saved_tensors
        N, H = weight.shape
        rows = _flat(dy, N)
        dx = torch.matmul(rows, weight).reshape(ctx.shape) if ctx.needs_input_grad[0] else None
        dw = None
        if ctx.needs_input_grad[1]:
            record = body.Act8Record(rows.shape[0], H, ctx.format, buffer=buffer)
            op = body.Act8WeightGrad(rows.shape[0], N, H, dtype=weight.dtype, device=dy.device)
            dw = op.run(rows, record)
            if ctx.sync_status:
                code, detail = op.status()
                if code != 0:
                    raise B.KdklError(code, f"device status of an act8_linear step, detail {detail}")
            else:
                _watch(op.workspace, "act8_linear")
        return dx, dw, None, None, None, None


def act8_linear(x, weight, record: Optional[body.Act8Record] = None, act8: str = "int8",
                sync_status: bool = False) -> torch.Tensor:
    """x @ weight.T (bf16, x [..., H], weight [N, H]) that keeps x in 8 bits for the weight's gradient: in `record`, if
    one that stands for x exists already (block_norm and gated_act leave them), else in one of format `act8`. A wait that
    runs out in the weight gradient's kernel is reported as the loss reports its steps: by check_status, by a later
    step, or by the backward call itself with sync_status (which waits for the kernel)."""
    if x.dtype != torch.bfloat16 or weight.dtype != torch.bfloat16:
        raise TypeError(f"act8_linear: expected bf16, got {x.dtype} and {weight.dtype}")
    if act8 not in ("int8", "e4m3"):
        raise ValueError(f"act8_linear: expected a record format, got {act8!r}")
    return _Act8Linear.apply(x, weight, record, act8, _recorded(weight), bool(sync_status))


class _GatedAct(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gate_up, act, act8, keep_h, needed):
        F = gate_up.shape[-1] // 2
        rows = _flat(gate_up, 2 * F)
        op = body.GatedAct(rows.shape[0], F, act=act, act8=act8 if needed else None, dtype=gate_up.dtype,
                           keep_h=keep_h and needed, device=gate_up.device)
        h = _shaped(op.forward(rows[:, :F], rows[:, F:]), (*gate_up.shape[:-1], F))
        if needed:
            ctx.save_for_backward(op.gate_record.buffer, op.up_record.buffer)   # autograd frees them, layer by layer
        record, op.h, op.h_record, op.gate_record, op.up_record = op.h_record, None, None, None, None
        ctx.op, ctx.shape, ctx.format = op, gate_up.shape, act8
        return h, record

    @staticmethod
    @_first_derivative_only("gated_act")
    def backward(ctx, dh, _):
        op, F = ctx.op, ctx.shape[-1] // 2
        op.gate_record, op.up_record = (body.Act8Record(op.T, F, ctx.format, buffer=b) for b in ctx.saved_tensors)
        op.dgate_up = None                                                      # a buffer of its own for every backward
        op.backward(_flat(dh, F))
        out, op.dgate_up, op.halves, op.gate_record, op.up_record = op.dgate_up, None, None, None, None
        return out.reshape(ctx.shape), None, None, None, None


def gated_act(gate_up, act: str = "silu", act8: str = "int8", keep_h: bool = False):
    """act(gate) * up of a projection [..., 2 F] whose first half is the gate; the backward pass reads both halves from
    8-bit records. With keep_h: (h, record of h), for the act8_linear that reads h."""
    if gate_up.shape[-1] % 2:
        raise TypeError(f"gated_act: expected an even width, got {gate_up.shape[-1]}")
    if act8 not in ("int8", "e4m3"):
        raise ValueError(f"gated_act: expected a record format, got {act8!r}")
    h, record = _GatedAct.apply(gate_up, act, act8, keep_h, _recorded(gate_up))
    return (h, record) if keep_h else h


class _BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, residual, branch, post_weight, pre_weight, gate, kind, act8, keep_y, args, train):
        H = branch.shape[-1]
        r, b = _flat(residual, H), _flat(branch, H)
        op = body.BlockNorm(b.shape[0], H, dtype=branch.dtype, residual_dtype=residual.dtype, gate=kind, act8=act8,
                            train=train, keep_y=keep_y, device=branch.device, **args)
        flat_gate = None if gate is None else gate.reshape(-1).contiguous()
        y, x = op.forward(r, b, post_weight=post_weight, pre_weight=pre_weight, gate=flat_gate)
        ctx.shapes = residual.shape, branch.shape, None if gate is None else gate.shape
        y, x = None if y is None else _shaped(y, branch.shape), _shaped(x, residual.shape)
        if train:
            # the branch and the sum, as records or as they are: autograd frees them layer by layer and, for tensors, checks
            # that nobody has changed them in place
            kept = (b, x) if act8 is None else (op.branch_record.buffer, op.sum_record.buffer)
            ctx.save_for_backward(post_weight, pre_weight, flat_gate, *kept)
        record = op.y_record
        op.kept = op.y = op.sum = op.y_record = op.branch_record = op.sum_record = None
        ctx.op, ctx.format = op, act8
        ctx.set_materialize_grads(False)
        return y, x, record

    @staticmethod
    @_first_derivative_only("block_norm")
    def backward(ctx, dy, dx, _):
        if dy is None and dx is None:
            return (None,) * 10
        op, (post_weight, pre_weight, gate, b, x) = ctx.op, ctx.saved_tensors
        rs, bs, gs = ctx.shapes
        H = bs[-1]
        if dy is None and pre_weight is not None:
            dy = torch.zeros(op.T, H, dtype=op.dtype, device=op.rho.device)
        if ctx.format is not None:
            op.branch_record, op.sum_record = (body.Act8Record(op.T, H, ctx.format, buffer=t) for t in (b, x))
        op.kept = (b, x if ctx.format is not None else _flat(x, H), post_weight, pre_weight, gate)
        op.workspace, op.grads = None, {}                                       # buffers of its own for every backward
        d = op.backward(None if dy is None else _flat(dy, H), None if dx is None else _flat(dx, H))
        op.kept = op.workspace = op.dresidual = op.dbranch = op.branch_record = op.sum_record = None
        return (d.residual.reshape(rs), d.branch.reshape(bs), d.post_weight, d.pre_weight,
                None if d.gate is None else d.gate.reshape(gs), None, None, None, None, None)


def block_norm(residual, branch, post_weight=None, pre_weight=None, gate=None, *, gate_kind: Optional[str] = None,
               act8: Optional[str] = None, keep_y: bool = False, eps: float = 1e-6, weight_offset: float = 0.0,
               branch_scale: float = 1.0, residual_scale: float = 1.0):
    """The join between two blocks (see body.BlockNorm): (y, x), y None without a pre_weight; with keep_y also the record
    of y for the act8_linear that reads it. The gate is one per channel if its shape is [H], else one per token; gate_kind
    says so where both fit. With act8 the backward pass reads 8-bit records of branch and x instead of the tensors."""
    if residual.shape != branch.shape:
        raise TypeError(f"block_norm: residual {tuple(residual.shape)} and branch {tuple(branch.shape)} differ")
    if gate is None:
        gate_kind = "none"
    elif gate_kind is None:
        lead = branch.shape[:-1]
        gate_kind = "channel" if gate.shape == branch.shape[-1:] else "token"
        if gate_kind == "token" and gate.dim() > 1 and gate.shape[-1] == gate.numel() == branch.shape[-1] \
                and gate.shape not in (lead, (*lead, 1)):
            raise TypeError(f"block_norm: a gate of shape {tuple(gate.shape)} beside a branch of {tuple(branch.shape)}: give it one "
                            "dimension if it is one per channel, or say gate_kind")
    if keep_y and (act8 is None or pre_weight is None):
        raise ValueError("block_norm: keep_y needs act8 and a pre_weight")
    args = dict(eps=eps, weight_offset=weight_offset, branch_scale=branch_scale, residual_scale=residual_scale)
    y, x, record = _BlockNorm.apply(residual, branch, post_weight, pre_weight, gate, gate_kind, act8, keep_y, args,
                                    _recorded(residual, branch, post_weight, pre_weight, gate))
    return (y, x, record) if keep_y else (y, x)


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, out_dtype, act8, keep_y, eps, train):
        H = x.shape[-1]
        rows = _flat(x, H)
        op = body.LayerNorm(rows.shape[0], H, dtype=out_dtype, x_dtype=x.dtype, act8=act8, eps=eps, train=train,
                            keep_y=keep_y and train, device=x.device)
        y = _shaped(op.forward(rows, weight, bias), x.shape)
        if train:
            ctx.save_for_backward(weight, bias, rows if act8 is None else op.x_record.buffer)
        record = op.y_record
        op.kept = op.y = op.y_record = op.x_record = None
        ctx.op, ctx.format, ctx.shape = op, act8, x.shape
        return y, record

    @staticmethod
    @_first_derivative_only("layer_norm")
    def backward(ctx, dy, _):
        op, (weight, bias, x) = ctx.op, ctx.saved_tensors
        if ctx.format is not None:
            op.x_record, x = body.Act8Record(op.T, op.H, ctx.format, buffer=x), None
        op.kept = (x, weight, bias)
        op.workspace, op.dx, op.grads = None, None, {}                          # buffers of its own for every backward
        d = op.backward(_flat(dy, op.H))
        op.kept = op.workspace = op.dx = op.x_record = None
        return d.x.reshape(ctx.shape), d.weight, d.bias, None, None, None, None, None


def layer_norm(x, weight=None, bias=None, *, eps: float = 1e-5, out_dtype=None, act8: Optional[str] = None,
               keep_y: bool = False):
    """Layer norm over the last dimension (see body.LayerNorm); x may be fp32 with an out_dtype of its own. With act8 the
    backward pass reads an 8-bit record of x instead of x; with keep_y: (y, record of y), for the act8_linear that reads y."""
    if keep_y and act8 is None:
        raise ValueError("layer_norm: keep_y needs act8")
    y, record = _LayerNorm.apply(x, weight, bias, out_dtype or x.dtype, act8, keep_y, eps, _recorded(x, weight, bias))
    return (y, record) if keep_y else y


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, rope):
        ctx.save_for_backward(positions)
        ctx.rope = rope
        ctx.set_materialize_grads(False)
        out = _rotate(rope.forward, q, k, positions)
        return out if k is not None else out[0]

    @staticmethod
    @_first_derivative_only("rotary")
    def backward(ctx, dq, dk=None):
        positions, = ctx.saved_tensors
        if dq is None:                                                          # one of the two may have no gradient
            return (None, None if dk is None else _rotate(ctx.rope.backward, dk, None, positions)[0], None, None)
        return (*_rotate(ctx.rope.backward, dq, dk, positions), None, None)


def _rotate(turn, q, k, positions):
    """One call on [..., heads, D] tensors, into outputs of its own."""
    places = positions.reshape(-1).contiguous()

    def rows(t):
        t = t.reshape(-1, *t.shape[-2:])
        return t if t.stride(-1) == 1 else t.contiguous()
    flat = [None if t is None else rows(t) for t in (q, k)]
    out = [None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k)]
    turn(*flat, places, out=[None if t is None else t.view(f.shape) for t, f in zip(out, flat)])
    return tuple(out)


def rotary(q, k, positions, rope: body.Rotary):
    """(q, k) turned by their tokens' positions: q [..., heads, D], k [..., kv heads, D] or None (then q alone is returned),
    positions [...] of int32 or int64."""
    for t in (q, k):
        if t is not None and t.shape[:-2] != positions.shape:
            raise TypeError(f"rotary: positions {tuple(positions.shape)} beside heads of {tuple(t.shape)}")
    return _Rotary.apply(q, k, positions, rope)


def _words16(t: torch.Tensor) -> torch.Tensor:
    """Rows that start on 16 bytes, as the tensor cores' loads need them (a copy where they do not)."""
    return t if t.data_ptr() % 16 == 0 and (t.shape[0] <= 1 or t.stride(0) % 8 == 0) else t.clone(memory_format=torch.contiguous_format)


class _GatedLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, record, act, act8, keep_h, train, sync_status):
        H, F = weight.shape[1], weight.shape[0] // 2
        rows, w = _words16(_flat(x, H)), _words16(weight.contiguous())
        op = body.GatedLinear(rows.shape[0], H, F, act=act, act8=act8, train=train, keep_h=keep_h and train, device=x.device)
        h = _shaped(op.forward(rows, w), (*x.shape[:-1], F))
        _watch(op.head, "gated_linear")
        if train:
            if act8 is not None and record is None and ctx.needs_input_grad[1]:
                record = body.Act8Record(rows.shape[0], H, act8, device=x.device).store(rows)
            kept = (rows,) if act8 is None else (op.gate_record.buffer, op.up_record.buffer, None if record is None else record.buffer)
            ctx.save_for_backward(w, *kept)
            ctx.format, ctx.shape, ctx.sync_status = act8, x.shape, sync_status
        h_record = op.h_record
        op.h = op.kept = op.gate_record = op.up_record = op.h_record = None
        ctx.op = op
        return h, h_record

    @staticmethod
    @_first_derivative_only("gated_linear")
    def backward(ctx, dh, _):
        op, (weight, *kept), record = ctx.op, ctx.saved_tensors, None
        if ctx.format is None:
            op.kept = (kept[0], weight)
        else:
            op.kept = (None, weight)
            op.gate_record, op.up_record = (body.Act8Record(op.T, op.F, ctx.format, buffer=b) for b in kept[:2])
            record = None if kept[2] is None else body.Act8Record(op.T, op.H, ctx.format, buffer=kept[2])
        op.workspace = op.dgate_up = op.dx = op.dweight = None                  # buffers of its own for every backward
        dx, dw = op.backward(_words16(_flat(dh, op.F)), record, want_dx=ctx.needs_input_grad[0], want_dweight=ctx.needs_input_grad[1])
        if ctx.sync_status:
            code, detail = op.status()
            if code != 0:
                raise B.KdklError(code, f"device status of a gated_linear step, detail {detail}")
        else:
            _watch(op.workspace, "gated_linear")
        op.kept = op.workspace = op.dgate_up = op.dx = op.dweight = op.gate_record = op.up_record = op.last = None
        return None if dx is None else dx.reshape(ctx.shape), dw, None, None, None, None, None, None


def gated_linear(x, weight, act: str = "silu", act8: Optional[str] = None, record: Optional[body.Act8Record] = None,
                 keep_h: bool = False, sync_status: bool = False):
    """act(x @ Wg.T) * (x @ Wu.T) in one kernel (see body.GatedLinear); x [..., H] and the stacked weight [2 F, H] are bf16.
    With act8 the backward pass reads 8-bit records of gate and up and, for the weight, of x: `record`, if one that stands
    for x exists already (layer_norm and block_norm leave them), else its own; with keep_h also (h, record of h). Without,
    it keeps x and forms gate and up again. Waits that ran out are reported as act8_linear reports them."""
    if x.dtype != torch.bfloat16 or weight.dtype != torch.bfloat16:
        raise TypeError(f"gated_linear: expected bf16, got {x.dtype} and {weight.dtype}")
    if weight.dim() != 2 or weight.shape[0] % 2 or weight.shape[1] != x.shape[-1]:
        raise TypeError(f"gated_linear: expected a weight [2 F, {x.shape[-1]}], got {tuple(weight.shape)}")
    if act8 not in (None, "int8", "e4m3"):
        raise ValueError(f"gated_linear: expected a record format or None, got {act8!r}")
    if keep_h and act8 is None:
        raise ValueError("gated_linear: keep_h needs act8")
    if record is not None and act8 is not None and (record.T, record.H, record.format) != (x.numel() // max(1, x.shape[-1]), x.shape[-1], act8):
        raise TypeError(f"gated_linear: the record is of {(record.T, record.H, record.format)}, the input of {tuple(x.shape)}, act8 {act8}")
    h, h_record = _GatedLinear.apply(x, weight, record, act, act8, keep_h, _recorded(x, weight), bool(sync_status))
    return (h, h_record) if keep_h else h


class _LabelLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, labels, token_weight, args, per_token, single_pass, train, sync_status):
        T, H, V = hidden.shape[0], hidden.shape[1], weight.shape[0]
        op = L.LabelLoss(T, H, V, train=train, device=hidden.device, **args)
        op.gradient_calls = (L._STEP,) if single_pass else (L._BACKWARD,)
        if single_pass and train:
            loss, dhidden, dweight = op.step(hidden, weight, labels, token_weight, want_dhidden=ctx.needs_input_grad[0],
                                             want_dweight=ctx.needs_input_grad[1])
            ctx.save_for_backward(dhidden, dweight)
        else:
            loss = op.forward(hidden, weight, labels, token_weight)
            if train:
                ctx.save_for_backward(hidden, weight, token_weight, op.state)
        out = op.losses.clone() if per_token else _shaped(loss, torch.Size(()))
        _settle(op, sync_status)
        op.workspaces, op.dhidden, op.dweight, op.losses, op.lse, op.loss, op.state, op.token_weight = {}, None, None, None, None, None, None, None
        ctx.op, ctx.per_token, ctx.done, ctx.sync_status = op, per_token, single_pass and train, sync_status
        return out

    @staticmethod
    @_first_derivative_only("label_loss")
    def backward(ctx, grad):
        op = ctx.op
        if ctx.done:                           # the gradients are there, for an upstream gradient of 1
            factor = grad.detach().to(torch.float32)
            return (*(None if t is None else L.rescaled(t, factor) for t in ctx.saved_tensors), None, None, None, None, None, None, None)
        hidden, weight, op.token_weight, op.state = ctx.saved_tensors
        op.args.state = op.state.data_ptr()
        dhidden, dweight = op.backward(hidden, weight, grad.detach().to(torch.float32).contiguous(), per_token=ctx.per_token,
                                       want_dhidden=ctx.needs_input_grad[0], want_dweight=ctx.needs_input_grad[1])
        _settle(op, ctx.sync_status)
        op.workspaces, op.dhidden, op.dweight, op.state, op.token_weight = {}, None, None, None, None
        return dhidden, dweight, None, None, None, None, None, None, None


def _settle(op, sync_status):
    if sync_status:
        code, detail = op.status()
        if code not in (0, -10):               # -10: labels out of range were ignored
            raise B.KdklError(code, f"device status of a label_loss step, detail {detail}")
    else:
        _watch(op.state, "label_loss")


def label_loss(hidden, weight, labels, token_weight: Optional[torch.Tensor] = None, *, ignore_index: int = -100,
               label_smoothing: float = 0.0, z_loss: float = 0.0, temperature: float = 1.0, reduction: str = "mean", chunk: int = 0,
               single_pass: bool = False, sync_status: bool = False) -> torch.Tensor:
    """Cross entropy of softmax(hidden @ weight.T / temperature) against labels [...] (int32 or int64), hidden [..., H] and weight
    [V, H] bf16 (see labels.LabelLoss for the formula). reduction "none" gives the losses [...], 0 at ignored tokens, without
    token weights. single_pass computes the gradients in the forward call, for an upstream gradient of 1 (three
    projections for four), and keeps them; another one then scales them, with one more rounding. Hidden states of ignored tokens
    have to be finite: they take part in dweight's product, with zeros."""
    if hidden.dtype != torch.bfloat16 or weight.dtype != torch.bfloat16:
        raise TypeError(f"label_loss: expected bf16, got {hidden.dtype} and {weight.dtype}")
    if hidden.shape[:-1] != labels.shape or (token_weight is not None and token_weight.shape != labels.shape):
        raise TypeError(f"label_loss: hidden {tuple(hidden.shape)} beside labels {tuple(labels.shape)}")
    if token_weight is not None and token_weight.requires_grad:
        raise TypeError("label_loss: token weights get no gradient: detach them, or weigh the losses of reduction \"none\"")
    if reduction not in ("mean", "sum", "none"):
        raise ValueError(f"label_loss: expected a reduction, got {reduction!r}")
    if reduction == "none" and (token_weight is not None or single_pass):
        raise ValueError("label_loss: the losses come without token weights and not in a single pass")
    args = dict(ignore_index=ignore_index, label_smoothing=label_smoothing, z_loss=z_loss, temperature=temperature, chunk=chunk,
                reduction="sum" if reduction == "none" else reduction)
    flat = [None if t is None else t.reshape(-1).contiguous() for t in (labels, token_weight)]
    out = _LabelLoss.apply(_words16(hidden.reshape(-1, hidden.shape[-1]).contiguous()), _words16(weight.contiguous()), *flat, args,
                           reduction == "none", bool(single_pass), _recorded(hidden, weight), bool(sync_status))
    return out.reshape(labels.shape) if reduction == "none" else out
