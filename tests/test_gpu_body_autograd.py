"""The student-body layers through autograd, and the example that runs them together.

Tolerances. Against torch's float64 autograd of the same layers on the tensors as given, the gradients carry the 8-bit
records' error. An int8 record's step is at most max/63.5 and its error uniform: at most max/127/sqrt(3) rms; of 32 normal
values the largest is below 3.2 deviations in nearly all groups: 1.5 % of a deviation, and e4m3's 2^-4/sqrt(3) relative at
most: 3.6 %. A gradient that is linear in the kept values has that error relative to its terms, which do not cancel here by
more than a factor of two or three: 5 % (int8) and 12 % (e4m3) bound them. Without records only bf16 roundings are left:
2^-8 each, a few of them in a row: 2 %.
"""
import importlib.util
import os

import pytest
import torch

from paper_2608_03796_b200 import autograd as A
from paper_2608_03796_b200 import body

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
LIMIT = {None: 0.02, "int8": 0.05, "e4m3": 0.12}


def _randn(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(BF16).cuda()


def _off(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


def _leaves(*tensors):
    return [t.detach().requires_grad_(True) for t in tensors], [t.detach().double().requires_grad_(True) for t in tensors]


@pytest.mark.parametrize("act8", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", [(3, 70), (210,)])
def test_linear(act8, shape):
    H, N = 264, 136
    (x, w), (x64, w64) = _leaves(_randn(1, *shape, H), _randn(2, N, H, scale=H ** -0.5))
    dy = _randn(3, *shape, N)
    y = A.act8_linear(x, w, act8=act8)
    assert y.shape == (*shape, N) and y.dtype == BF16
    y.backward(dy)
    (x64 @ w64.t()).backward(dy.double())
    assert _off(x.grad, x64.grad) <= 0.01 and x.grad.shape == x.shape
    assert _off(w.grad, w64.grad) <= LIMIT[act8] and w.grad.dtype == BF16
    # exactly what the record stands for
    rec = body.Act8Record(210, H, act8).store(x.detach().reshape(-1, H))
    want = dy.double().reshape(-1, N).t() @ rec.load(dtype=torch.float32).double()
    assert _off(w.grad, want) <= 2.0 ** -8
    # a record that exists already is used: nothing of the input itself is read again
    other = body.Act8Record(210, H, act8).store(torch.zeros_like(x.detach().reshape(-1, H)))
    w.grad = None
    A.act8_linear(x.detach(), w, record=other).backward(dy)
    assert not w.grad.any()
    with pytest.raises(TypeError):
        A.act8_linear(x, w, record=body.Act8Record(209, H, act8))
    with pytest.raises(TypeError):
        A.act8_linear(x.float(), w)
    with pytest.raises(ValueError):
        A.act8_linear(x, w, act8=None)


@pytest.mark.parametrize("act8", ["int8", "e4m3"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated(act8, act):
    T, F = 130, 520
    (z,), (z64,) = _leaves(_randn(1, 2, T // 2, 2 * F, scale=1.5))
    dh = _randn(2, 2, T // 2, F)
    h, rec = A.gated_act(z, act=act, act8=act8, keep_h=True)
    g64, u64 = z64.chunk(2, dim=-1)
    f = torch.nn.functional
    h64 = (f.silu(g64) if act == "silu" else f.gelu(g64, approximate="tanh")) * u64
    assert h.shape == h64.shape and _off(h.detach(), h64.detach()) <= 2.0 ** -8
    assert torch.equal(rec.load(), body.Act8Record(T, F, act8).store(h.detach().reshape(T, F)).load())
    h.backward(dh)
    h64.backward(dh.double())
    assert _off(z.grad, z64.grad) <= LIMIT[act8]
    with torch.no_grad():
        h2 = A.gated_act(z, act=act, act8=act8)
    assert torch.equal(h2, h.detach())
    with pytest.raises(TypeError):
        A.gated_act(z[..., :-1])


@pytest.mark.parametrize("act8", [None, "int8", "e4m3"])
@pytest.mark.parametrize("kind", ["none", "channel", "token"])
def test_block_norm(act8, kind):
    shape, H = (3, 50), 264
    tensors = [_randn(1, *shape, H), _randn(2, *shape, H), 1 + _randn(3, H, scale=0.1), 1 + _randn(4, H, scale=0.1)]
    if kind != "none":
        tensors.append(0.5 + _randn(5, *((H,) if kind == "channel" else (*shape, 1)), scale=0.2))
    ours, theirs = _leaves(*tensors)
    dy, dx = _randn(6, *shape, H), _randn(7, *shape, H)
    y, x = A.block_norm(*ours[:4], ours[4] if kind != "none" else None, act8=act8, eps=1e-5, branch_scale=0.5,
                        residual_scale=1.25)
    r, b, w1, w2 = theirs[:4]
    gate = theirs[4] if kind != "none" else 1.0

    def rms(v):
        return torch.rsqrt((v * v).mean(-1, keepdim=True) + 1e-5)
    x64 = 1.25 * r + 0.5 * gate * (b * rms(b) * w1)
    y64 = x64 * rms(x64) * w2
    assert _off(y.detach(), y64.detach()) <= 2.0 ** -8 and _off(x.detach(), x64.detach()) <= 2.0 ** -8
    torch.autograd.backward([y, x], [dy, dx])
    torch.autograd.backward([y64, x64], [dy.double(), dx.double()])
    for got, want in zip(ours, theirs):
        assert got.grad.shape == want.shape and got.grad.dtype == BF16
        assert _off(got.grad, want.grad) <= LIMIT[act8]
    # the residual stream alone, and y alone
    for outs, grads, outs64 in (((x,), (dx,), (x64,)), ((y,), (dy,), (y64,))):
        for t in (*ours, *theirs):
            t.grad = None
        y2, x2 = A.block_norm(*ours[:4], ours[4] if kind != "none" else None, act8=act8, eps=1e-5, branch_scale=0.5,
                              residual_scale=1.25)
        x64 = 1.25 * r + 0.5 * gate * (b * rms(b) * w1)
        y64 = x64 * rms(x64) * w2
        (x2 if outs[0] is x else y2).backward(grads[0])
        (x64 if outs[0] is x else y64).backward(grads[0].double())
        assert _off(ours[0].grad, theirs[0].grad) <= LIMIT[act8] and _off(ours[1].grad, theirs[1].grad) <= LIMIT[act8]


def test_broadcast_gate_and_expanded_gradients():
    """A scalar gate that its owner expands gets the sum over what it was broadcast to; gradients with zero strides (of
    a sum) are taken as they are."""
    T, H = 40, 96
    r, b = _randn(1, T, H), _randn(2, T, H)
    gate = torch.tensor(0.3, dtype=BF16, device="cuda", requires_grad=True)
    y, x = A.block_norm(r, b, gate=gate.expand(H))
    assert y is None
    x.sum().backward()
    want = b.double().sum().item()
    assert abs(gate.grad.item() - want) <= 2.0 ** -7 * b.double().abs().sum().item() ** 0.5 * 4 + 2.0 ** -7 * abs(want)


def test_saved_state_is_autograds():
    """Two graphs at once, a second backward through a retained graph, a change in place of what was kept, hooks that move
    saved tensors, and no state kept where nothing needs a gradient."""
    T, H = 64, 128
    r, b, w = _randn(1, T, H).requires_grad_(True), _randn(2, T, H).requires_grad_(True), torch.ones(H, dtype=BF16, device="cuda")
    dy = _randn(3, T, H)

    def grads(act8, twice=False):
        r.grad = b.grad = None
        y, x = A.block_norm(r, b, w, w, act8=act8)
        y2, _ = A.block_norm(r * 2, b * 3, w, w, act8=act8)                  # another graph of the shape, alive in between
        y.backward(dy, retain_graph=twice)
        if twice:
            y.backward(dy)
        return r.grad.clone(), b.grad.clone()
    for act8 in (None, "int8"):
        once, twice = grads(act8), grads(act8, True)
        assert all(torch.equal(2 * a, c) for a, c in zip(once, twice))

        def to_host(t):
            return t.cpu()

        def to_device(t):
            return t.cuda()
        with torch.autograd.graph.saved_tensors_hooks(to_host, to_device):
            moved = grads(act8)
        assert all(torch.equal(a, c) for a, c in zip(once, moved))
    y, x = A.block_norm(r, b, w, w)
    x.add_(1.0)
    with pytest.raises(RuntimeError):
        y.backward(dy)
    with torch.no_grad():
        y, x, rec = A.block_norm(r, b, w, w, act8="int8", keep_y=True)
    assert rec is None
    with pytest.raises(ValueError):
        A.block_norm(r, b, w, w, keep_y=True)
    with pytest.raises(TypeError):
        A.block_norm(r, b[:, :64], w, w)


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "student_step.py")
    spec = importlib.util.spec_from_file_location("student_step", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("act8", [None, "int8", "e4m3"])
def test_example_step_against_float64(act8):
    """One step of the example, loss and every parameter's gradient against float64 autograd of the same student. A
    gradient passes two blocks' records on its way, so twice the layer's limit holds for it."""
    E = _example()
    T, H, F, V, K = 200, 128, 264, 512, 8
    student = E.Student(H, F, V, layers=2)
    x = _randn(1, T, H)
    g = torch.Generator().manual_seed(5)
    idx = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)]).to(torch.int32).cuda()
    val = (3 * torch.randn(T, K, generator=g)).cuda()
    loss = E.step(student, x, (idx, val), act8, chunk=64)
    A.check_status()
    p = {n: t.detach().double().requires_grad_(True) for n, t in student.named_parameters()}

    def rms(v):
        return torch.rsqrt((v * v).mean(-1, keepdim=True) + 1e-5)
    r = x.double()
    y = r * rms(r) * p["first"]
    for n in range(2):
        gate, up = (y @ p[f"blocks.{n}.gate_up"].t()).chunk(2, dim=-1)
        b = (torch.nn.functional.silu(gate) * up) @ p[f"blocks.{n}.down"].t()
        r = r + 0.5 * p[f"blocks.{n}.gate"] * (b * rms(b) * p[f"blocks.{n}.post"])
        y = r * rms(r) * p[f"blocks.{n}.pre"]
    logits = y @ p["head"].t()
    t = torch.softmax(val.double(), dim=1)
    want = (t * (t.log() - torch.gather(logits, 1, idx.long()) + torch.logsumexp(logits, 1, keepdim=True))).sum(1).mean()
    want.backward()
    assert abs(loss.item() - want.item()) <= 5e-3 * abs(want.item())
    for n, q in student.named_parameters():
        assert _off(q.grad, p[n].grad) <= 2 * LIMIT[act8], n
