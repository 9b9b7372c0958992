"""The label loss on the GPU against its formulas in 64 bits.

Tolerances. A logit is off by ez = (H / 16 + 16) 2^-23 sum |h||w| / tau (the tensor cores add 16 products at a time, each addition
cutting at most a unit off). The normaliser moves by as much, and by 2^-20 relative in the exponentials and the sums of 256-column
tiles: a loss by (2 + 2 lambda |lse|) ez and 2^-20 of its parts. G is a q - c - b [v = y]: q is off by 2 ez + 2^-19 relative, and in
one pass by an fp16 rounding (2^-11) or, 2^-14 and more below the largest of its 32 columns, 2^-25 of that; the sum is rounded to
bf16, whose 8 significant bits make neighbours 2^-7 of the lower end of their binade apart: off by at most 2^-8 of the value.
dhidden and dweight are sums of G times exact numbers, in fp32 (n / 16 + 16 units), and rounded once to their type. (The value
that is rounded is the computed one, which the terms' errors are part of.) Over many values the roundings have no preferred
sign: the norm of the difference is at most 3.2e-3 of the result's (an error spread evenly over half a step either way has a
root mean square of 2^-8 / sqrt 3 at the lower end of a binade and half that at the upper one, 1.7e-3 over it; two make 2.4e-3).
"""
import pytest
import torch

from paper_2608_03796_b200 import binding as B
from paper_2608_03796_b200.autograd import check_status, fused_chunked_kl, label_loss
from paper_2608_03796_b200.labels import LabelLoss

pytestmark = pytest.mark.gpu
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
IGNORED = -100


def _unit(n):
    return (n / 16 + 16) * 2.0 ** -23


def _inputs(T, H, V, seed=0, ignored=0.2, scale=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = (scale * torch.randn(T, H, generator=g, device="cuda")).to(BF16)
    w = (torch.randn(V, H, generator=g, device="cuda") / H ** 0.5).to(BF16)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    y[torch.rand(T, generator=g, device="cuda") < ignored] = IGNORED
    return h, w, y, 2 * torch.rand(T, generator=g, device="cuda")


class _Want:
    def __init__(self, h, w, y, s=0.0, lam=0.0, tau=1.0):
        self.h, self.w, self.s, self.lam, self.tau = h.double(), w.double(), s, lam, tau
        T, V = len(h), len(w)
        z = self.h @ self.w.t() / tau
        self.ez = (_unit(h.shape[1]) * (self.h.abs() @ self.w.abs().t()) / tau).amax(1)
        self.counted = (y >= 0) & (y < V)
        self.col = torch.where(self.counted, y, torch.zeros_like(y))[:, None]
        self.lse = torch.logsumexp(z, 1)
        zy = z.gather(1, self.col)[:, 0]
        zero = torch.zeros_like(zy)
        self.losses = torch.where(self.counted, self.lse - (1 - s) * zy - s * z.mean(1) + lam * self.lse ** 2, zero)
        self.slack = torch.where(self.counted, (2 + 2 * lam * self.lse.abs()) * self.ez + 2.0 ** -20 * (
            1 + self.lse.abs() + zy.abs() + s * z.abs().mean(1) + lam * self.lse ** 2), zero)
        self.q = torch.softmax(z, 1)
        top = torch.nn.functional.pad(self.q, (0, -V % 32)).reshape(T, -1, 32).amax(-1, keepdim=True).expand(-1, -1, 32)
        self.top = top.reshape(T, -1)[:, :V]

    def grads(self, g):
        """G, its bound, and dhidden and dweight with theirs; g [T]: upstream gradient of the losses."""
        g = (g.double() * self.counted)[:, None] / self.tau
        a = g * (1 + 2 * self.lam * self.lse)[:, None]
        G = a * self.q - g * self.s / len(self.w)
        G.scatter_add_(1, self.col, -(1 - self.s) * g)
        bound = a.abs() * (self.q * (2 * self.ez[:, None] + 2.0 ** -19 + 2.0 ** -11) + self.top * 2.0 ** -25)
        bound += a.abs() * self.q * (2 * self.lam * self.ez)[:, None] + 2.0 ** -22 * (g.abs() + a.abs()) * (self.q + self.s / len(self.w))
        bound = bound.scatter_add(1, self.col, 2.0 ** -22 * g.abs())
        bound = bound * (1 + 2.0 ** -8) + G.abs() * 2.0 ** -8
        dh, dw = G @ self.w, G.t() @ self.h
        return ((dh, bound @ self.w.abs() + _unit(len(self.w)) * (G.abs() @ self.w.abs())),
                (dw, bound.t() @ self.h.abs() + _unit(len(self.h)) * (G.abs().t() @ self.h.abs())))


def _near(got, want, slack, what, many=False):
    t = torch.finfo(got.dtype)
    bad = (got.double() - want).abs() - ((want.abs() + slack) * (t.eps / 2) + t.smallest_normal + slack)
    assert torch.isfinite(got).all() and float(bad.max()) <= 0, f"{what}: {float(bad.max())} beyond the bound"
    if many:
        off = float((got.double() - want).norm() / want.norm())
        assert off <= 3.2e-3, f"{what}: {off} in norm"


def _check_grads(want, g, dh, dw, many=False):
    for got, (value, slack), name in zip((dh, dw), want.grads(g), ("dhidden", "dweight")):
        _near(got, value, slack, name, many)
    assert not dh[~want.counted].any()                                      # exact zeros


def _check_loss(want, op, weight=None, divisor=None):
    w = want.counted.double() if weight is None else want.counted * weight.double()
    d = max(1.0, float(want.counted.sum())) if divisor is None else divisor
    _near(op.losses, want.losses, want.slack, "losses")
    _near(op.loss, ((want.losses * w).sum() / d).reshape(1), ((want.slack * w.abs()).sum() / d).reshape(1), "loss")
    assert not op.losses[~want.counted].any() and not op.lse[~want.counted].any()
    _near(op.lse[want.counted], want.lse[want.counted], (want.ez + 2.0 ** -20 * (1 + want.lse.abs()))[want.counted], "lse") if want.counted.any() else None
    return w / d


# up to 128 tokens (each width of the narrow tile; ragged last tiles; more tiles than SMs), and more
SHAPES = [(1, 8, 1), (1, 64, 7), (2, 2048, 9001), (3, 64, 1000), (16, 72, 128), (17, 512, 40001), (33, 64, 161), (64, 264, 20002),
          (65, 1000, 33), (128, 128, 30000), (129, 128, 2000), (257, 128, 515), (300, 264, 2001), (700, 512, 4096)]


@pytest.mark.parametrize("T,H,V", SHAPES)
@pytest.mark.parametrize("s,lam,tau", [(0.0, 0.0, 1.0), (0.1, 0.0, 1.0), (0.0, 1e-3, 2.0), (0.3, 1e-2, 0.5)])
def test_two_calls_and_one_step(T, H, V, s, lam, tau):
    h, w, y, weight = _inputs(T, H, V, seed=T + V)
    want = _Want(h, w, y, s, lam, tau)
    op = LabelLoss(T, H, V, label_smoothing=s, z_loss=lam, temperature=tau)
    many = T >= 256
    for token_weight in (None, weight):
        op.forward(h, w, y, token_weight)
        g = _check_loss(want, op, token_weight)
        _check_grads(want, g, *op.backward(h, w), many=many)
        op.loss.zero_(), op.losses.zero_(), op.dhidden.fill_(7), op.dweight.fill_(7)
        _, dh, dw = op.step(h, w, y, token_weight)
        _check_loss(want, op, token_weight)
        _check_grads(want, g, dh, dw, many=many)
    assert op.status()[0] == 0 and op.status()[1][1] == int(want.counted.sum())


@pytest.mark.parametrize("chunk", [1, 256, 300, 512])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_chunks(chunk, dtype):
    """Several chunks, the last one short, one of them with no counted token; fp32 gradients and int32 labels."""
    T, H, V = 1100, 128, 777
    h, w, y, weight = _inputs(T, H, V)
    y[256:530] = IGNORED
    want = _Want(h, w, y, 0.1, 1e-3)
    op = LabelLoss(T, H, V, label_smoothing=0.1, z_loss=1e-3, chunk=chunk, dtype=dtype, dhidden_dtype=dtype, reduction="sum")
    op.forward(h, w, y.int(), weight)
    g = _check_loss(want, op, weight, divisor=1.0)
    _check_grads(want, g, *op.backward(h, w), many=True)
    op.dhidden.fill_(7), op.dweight.fill_(7)
    _, dh, dw = op.step(h, w, y.int(), weight)
    _check_grads(want, g, dh, dw, many=True)


def test_upstream_gradients():
    """A number on the device, of either sign; one a token, of both signs and zeros; a divisor from elsewhere."""
    T, H, V = 300, 128, 1000
    h, w, y, _ = _inputs(T, H, V)
    want = _Want(h, w, y, 0.1, 1e-3)
    divisor = torch.tensor([1234.0], dtype=F64, device="cuda")
    op = LabelLoss(T, H, V, label_smoothing=0.1, z_loss=1e-3, denom_device=divisor)
    op.forward(h, w, y)
    g = _check_loss(want, op, divisor=1234.0)
    up = torch.tensor([-3.0], device="cuda")
    _check_grads(want, -3 * g, *op.backward(h, w, up), many=True)
    _check_grads(want, -3 * g, *op.step(h, w, y, grad=up)[1:], many=True)
    each = torch.randn(T, device="cuda")
    each[::7] = 0
    _check_grads(want, each, *op.backward(h, w, each), many=True)


def test_a_gradient_that_is_added():
    T, H, V = 600, 128, 333
    h, w, y, _ = _inputs(T, H, V)
    want = _Want(h, w, y)
    for chunk in (0, 256):
        op = LabelLoss(T, H, V, dtype=F32, chunk=chunk, reduction="sum")
        total = torch.ones(V, H, device="cuda")
        _, dh, dw = op.step(h, w, y, out=total, accumulate=True)
        value, slack = want.grads(torch.ones(T, device="cuda"))[1]
        assert dw is total
        _near(total, value + 1, slack + 2.0 ** -22 * (1 + value.abs()), "1 + dweight")
    with pytest.raises(B.KdklError):
        LabelLoss(T, H, V).step(h, w, y, accumulate=True)


def test_a_frozen_head_or_frozen_hidden_states():
    T, H, V = 300, 64, 500
    h, w, y, _ = _inputs(T, H, V)
    op = LabelLoss(T, H, V)
    _, dh, dw = (t.clone() for t in op.step(h, w, y))
    assert torch.equal(op.step(h, w, y, want_dweight=False)[1], dh) and torch.equal(op.step(h, w, y, want_dhidden=False)[2], dw)
    assert op.step(h, w, y, want_dweight=False)[2] is None
    op.forward(h, w, y)
    both = [t.clone() for t in op.backward(h, w)]
    assert torch.equal(op.backward(h, w, want_dweight=False)[0], both[0]) and torch.equal(op.backward(h, w, want_dhidden=False)[1], both[1])
    for single_pass in (False, True):
        a, b = h.clone().requires_grad_(), w.clone().requires_grad_()
        label_loss(a, w, y, single_pass=single_pass).backward()
        label_loss(h, b, y, single_pass=single_pass).backward()
        for got, want in ((a.grad, dh if single_pass else both[0]), (b.grad, dw if single_pass else both[1])):
            assert torch.equal(got, want)
    with pytest.raises(ValueError):
        op.step(h, w, y, want_dhidden=False, want_dweight=False)


def test_nothing_counted_and_labels_out_of_range():
    T, H, V = 300, 64, 100
    h, w, y, _ = _inputs(T, H, V)
    op = LabelLoss(T, H, V)
    for call in (lambda: op.step(h, w, torch.full_like(y, IGNORED)), lambda: (op.forward(h, w, torch.full_like(y, IGNORED)), *op.backward(h, w))):
        loss, dh, dw = call()
        assert loss.item() == 0 and not dh.any() and not dw.any() and not op.losses.any() and op.status()[0] == 0
    bad = y.clone()
    bad[3], bad[4], bad[5] = V, -1, 1 << 40
    want = _Want(h, w, bad)
    _, dh, dw = op.step(h, w, bad)
    _check_grads(want, _check_loss(want, op), dh, dw, many=True)
    code, detail = op.status()
    assert code == -10 and detail[2] == 3 and detail[1] == int(want.counted.sum())
    zero = LabelLoss(0, H, V)
    loss, dh, dw = zero.step(h[:0], w, y[:0])
    assert loss.item() == 0 and dh.shape == (0, H) and not dw.any()
    other = LabelLoss(T, H, V, ignore_index=5)                              # an index that is a column as well
    y5 = torch.where(y < 0, torch.full_like(y, 5), y)
    other.forward(h, w, y5)
    _check_loss(_Want(h, w, torch.where(y5 == 5, torch.full_like(y, -1), y5)), other)


def test_logits_far_from_zero():
    """One pass keeps exponentials relative to their neighbours' largest: logits near 1000, near -1000 and 2000 apart are no
    special case. The logits are exact here (one column of the hidden states, powers of two)."""
    T, H, V = 6, 8, 300
    h = torch.zeros(T, H, dtype=BF16, device="cuda")
    w = torch.zeros(V, H, dtype=BF16, device="cuda")
    h[:, 0], h[:, 1] = torch.tensor([1.0, 1.0, 0.0, 64.0, -64.0, 0.25]).to(BF16).cuda(), 1.0
    w[:, 0] = torch.randn(V, device="cuda").to(BF16)
    for shift in (-1000.0, 0.0, 1000.0):
        w[:, 1] = shift
        y = torch.tensor([0, 299, 5, 7, 9, IGNORED], device="cuda")
        want = _Want(h, w, y)
        op = LabelLoss(T, H, V)
        _, dh, dw = op.step(h, w, y)
        assert op.status()[0] == 0
        _check_grads(want, _check_loss(want, op), dh, dw)


def test_a_state_of_another_call_is_refused_on_the_device():
    T, H, V = 600, 64, 200
    h, w, y, _ = _inputs(T, H, V)
    op = LabelLoss(T, H, V)
    op.forward(h, w, y)
    other = LabelLoss(T, H, V, chunk=256)
    other.fed = True
    other.state.copy_(op.state)
    other._outputs(None, False)
    other.dhidden.fill_(7), other.dweight.fill_(7)
    dh, dw = other.backward(h, w)
    assert other.status()[0] == -9 and (dh == 7).all() and (dw == 7).all()


def test_the_same_every_time_and_captured():
    T, H, V = 500, 128, 1500
    h, w, y, weight = _inputs(T, H, V)
    op = LabelLoss(T, H, V, label_smoothing=0.1)
    first = [t.clone() for t in op.step(h, w, y, weight)]
    assert all(torch.equal(a, b) for a, b in zip(first, op.step(h, w, y, weight)))
    op.forward(h, w, y, weight), op.backward(h, w)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            loss, dh, dw = op.step(h, w, y, weight)
            one = [t.clone() for t in (loss, dh, dw)]
            op.forward(h, w, y, weight)
            dh, dw = op.backward(h, w)
        h2, _, y2, _ = _inputs(T, H, V, seed=8)
        h.copy_(h2), y.copy_(y2)
        graph.replay()
    torch.cuda.synchronize()
    want = _Want(h, w, y, 0.1)
    g = _check_loss(want, op, weight)
    _check_grads(want, g, dh, dw, many=True)
    _check_grads(want, g, one[1], one[2], many=True)


@pytest.mark.parametrize("single_pass", [False, True])
def test_autograd(single_pass):
    """Leading dimensions; an upstream gradient that is not 1; against differences of the formula in 64 bits along a random
    direction: the inner product is off by the roundings' share of the gradient's norm."""
    T, H, V = 240, 64, 500
    h, w, y, weight = _inputs(T, H, V)
    a, b = h.reshape(2, 120, H).clone().requires_grad_(), w.clone().requires_grad_()
    loss = label_loss(a, b, y.reshape(2, 120), weight.reshape(2, 120), label_smoothing=0.1, z_loss=1e-3, single_pass=single_pass)
    (0.5 * loss).backward()
    check_status()
    n = (y >= 0).sum()

    def total(p, q):
        want = _Want(p, q, y, 0.1, 1e-3)
        return 0.5 * float((want.losses * weight.double() * want.counted).sum() / n)
    assert abs(0.5 * loss.item() - total(h, w)) <= 1e-5
    for t, grad, at in ((h, a.grad.reshape(T, H), 0), (w, b.grad, 1)):
        v = torch.randn(t.shape, dtype=F64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
        f = (lambda e: total(h.double() + e * v, w)) if at == 0 else (lambda e: total(h, w.double() + e * v))
        slope = (f(1e-4) - f(-1e-4)) / 2e-4
        assert abs(float((grad.double() * v).sum()) - slope) <= 0.02 * float(grad.double().norm()) + 1e-7


def test_losses_with_a_gradient_each():
    T, H, V = 100, 64, 300
    h, w, y, _ = _inputs(T, H, V)
    a, b = h.reshape(4, 25, H).clone().requires_grad_(), w.clone().requires_grad_()
    losses = label_loss(a, b, y.reshape(4, 25), reduction="none")
    assert losses.shape == (4, 25)
    up = torch.randn(4, 25, device="cuda")
    losses.backward(up, retain_graph=True)
    want = _Want(h, w, y)
    _check_grads(want, up.reshape(-1), a.grad.reshape(T, H), b.grad)
    first = a.grad.clone()
    a.grad = None
    losses.backward(up)                                                     # again through the same graph
    assert torch.equal(a.grad, first)
    one = label_loss(h[:1].clone().requires_grad_(), w, torch.tensor([3], device="cuda"), reduction="none")
    one.backward(torch.tensor([2.0], device="cuda"))
    with torch.no_grad():
        assert label_loss(h, w, y).item() > 0


def test_beside_the_loss_against_a_teacher():
    """Plain cross entropy is the KL loss against a teacher with one entry of probability 1."""
    T, H, V = 400, 128, 900
    h, w, y, _ = _inputs(T, H, V, ignored=0.0)
    a, b = label_loss(h, w, y), fused_chunked_kl(h, w, y.int()[:, None].contiguous(), torch.zeros(T, 1, device="cuda"))
    want = _Want(h, w, y)
    assert abs(float(a) - float(b)) <= 2 * float(want.slack.mean())


def test_refusals():
    T, H, V = 16, 64, 100
    h, w, y, weight = _inputs(T, H, V)
    op = LabelLoss(T, H, V)
    with pytest.raises(RuntimeError, match="before any forward"):
        op.backward(h, w)
    for bad in (lambda: op.forward(h.float(), w, y), lambda: op.forward(h, w[:50], y), lambda: op.forward(h, w, y[:8]),
                lambda: op.forward(h, w, y, weight.double()), lambda: op.forward(h.cpu(), w, y),
                lambda: op.step(h, w, y, grad=torch.ones(T, device="cuda")), lambda: label_loss(h, w, y[:8]),
                lambda: label_loss(h, w, y, weight.clone().requires_grad_()),
                lambda: label_loss(h.float(), w, y), lambda: op.forward(torch.zeros(T, 2 * H, dtype=BF16, device="cuda")[:, :H], w, y)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: op.forward(h, w, y.float()), lambda: label_loss(h, w, y, reduction="median"),
                lambda: label_loss(h, w, y, weight, reduction="none"), lambda: LabelLoss(T, 60, V), lambda: LabelLoss(T, H, V, label_smoothing=1.5)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RuntimeError, match="evaluation"):
        LabelLoss(T, H, V, train=False).step(h, w, y)
