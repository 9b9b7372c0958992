"""The operators of a student together, as a training step and a decoding step use them: layer norm, projections, rotary positions,
attention (plain torch), gated linear layer, label loss beside the loss against a teacher.

Tolerance of the chain's gradients against the same network in 64 bits: a bf16 rounding is off by 1.7e-3 of the value, root mean
square; some 20 of them lie between the loss and the first weight and back, without preferred sign, and a residual stream does not
amplify them: 20^(1/2) 1.7e-3 = 8e-3, taken three times. int8 records of x, gate, up and h add 1/254 sqrt(2) of a group's largest
value (2.1 deviations) each, 1.2e-2 of the value's size; four of them on the way: 2.4e-2 more, taken three times as well.
"""
import math

import pytest
import torch

from paper_2608_03796_b200 import autograd as A
from paper_2608_03796_b200 import body
from paper_2608_03796_b200.labels import LabelLoss

pytestmark = pytest.mark.gpu
BF16, F64 = torch.bfloat16, torch.float64
Bt, S, H, F, V, HEADS, KV, D = 2, 48, 128, 320, 700, 4, 2, 32


def _weights(seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def mat(n, k):
        return (torch.randn(n, k, generator=g, device="cuda") / k ** 0.5).to(BF16)
    w = dict(qkv=mat((HEADS + 2 * KV) * D, H), out=mat(H, HEADS * D), gate_up=mat(2 * F, H), down=mat(H, F), head=mat(V, H))
    for n in ("n1", "n2", "n3"):
        w[n] = (1 + 0.2 * torch.randn(H, generator=g, device="cuda")).to(BF16)
        w["b" + n] = (0.1 * torch.randn(H, generator=g, device="cuda")).to(BF16)
    x = torch.randn(Bt, S, H, generator=g, device="cuda").to(BF16)
    labels = torch.randint(0, V, (Bt, S), generator=g, device="cuda")
    labels[:, :5] = -100
    topk = torch.randint(0, V, (Bt * S, 8), generator=g, device="cuda", dtype=torch.int32)
    return w, x, labels, topk


def _attention(q, k, v):
    k, v = (t.repeat_interleave(HEADS // KV, dim=2) for t in (k, v))
    s = torch.einsum("bqhd,bkhd->bhqk", q, k) / math.sqrt(D)
    s = s.masked_fill(torch.ones(q.shape[1], k.shape[1], dtype=torch.bool, device="cuda").triu(1), -math.inf)
    return torch.einsum("bhqk,bkhd->bqhd", torch.softmax(s.float() if s.dtype == BF16 else s, -1).to(q.dtype), v)


def _step(w, x, labels, topk, rope, act8):
    """The loss of the student, all its own operators in play."""
    positions = torch.arange(S, device="cuda").expand(Bt, S)
    keep = dict(act8=act8, keep_y=True) if act8 else {}
    first = A.layer_norm(x, w["n1"], w["bn1"], **keep)
    y, kept = first if act8 else (first, None)
    qkv = A.act8_linear(y, w["qkv"], record=kept) if act8 else torch.nn.functional.linear(y, w["qkv"])
    q, k, v = qkv.reshape(Bt, S, -1, D).split((HEADS, KV, KV), dim=2)
    q, k = A.rotary(q, k, positions, rope)
    x = x + torch.nn.functional.linear(_attention(q, k, v).reshape(Bt, S, -1), w["out"])
    second = A.layer_norm(x, w["n2"], w["bn2"], **keep)
    y, kept = second if act8 else (second, None)
    if act8:
        h, kept = A.gated_linear(y, w["gate_up"], act8=act8, record=kept, keep_h=True)
        branch = A.act8_linear(h, w["down"], record=kept)
    else:
        branch = torch.nn.functional.linear(A.gated_linear(y, w["gate_up"]), w["down"])
    y = A.layer_norm(x + branch, w["n3"], w["bn3"])
    hard = A.label_loss(y, w["head"], labels, label_smoothing=0.1, z_loss=1e-3)
    soft = A.fused_chunked_kl(y.reshape(-1, H), w["head"], topk, torch.zeros(topk.shape, device="cuda"), chunk=64)
    return hard + 0.5 * soft


def _plain(w, x, labels, topk):
    """The same in 64 bits."""
    def norm(x, n):
        return torch.nn.functional.layer_norm(x, (H,), w[n], w["b" + n])
    f = 10000.0 ** (-2 * torch.arange(D // 2, dtype=F64, device="cuda") / D)
    angle = torch.arange(S, dtype=F64, device="cuda")[:, None, None] * f

    def turned(t):
        a, b = t[..., :D // 2], t[..., D // 2:]
        return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)
    q, k, v = (norm(x, "n1") @ w["qkv"].t()).reshape(Bt, S, -1, D).split((HEADS, KV, KV), dim=2)
    x = x + _attention(turned(q), turned(k), v).reshape(Bt, S, -1) @ w["out"].t()
    z = norm(x, "n2") @ w["gate_up"].t()
    x = x + (torch.nn.functional.silu(z[..., :F]) * z[..., F:]) @ w["down"].t()
    logits = (norm(x, "n3") @ w["head"].t()).reshape(-1, V)
    logp, counted = torch.log_softmax(logits, -1), labels.reshape(-1) >= 0
    lse = torch.logsumexp(logits, -1)
    hard = 0.9 * -logp.gather(1, labels.reshape(-1, 1).clamp(min=0))[:, 0] - 0.1 * logp.mean(-1) + 1e-3 * lse ** 2
    soft = -(logp.gather(1, topk.long()) / topk.shape[1]).sum(-1) - math.log(topk.shape[1])
    return hard[counted].mean() + 0.5 * soft.mean()


@pytest.mark.parametrize("act8,most", [(None, 0.024), ("int8", 0.1)])
def test_a_training_step(act8, most):
    w, x, labels, topk = _weights()
    for t in w.values():
        t.requires_grad_()
    x.requires_grad_()
    loss = _step(w, x, labels, topk, body.Rotary(D), act8)
    loss.backward()
    A.check_status()
    w64 = {n: t.detach().double().requires_grad_() for n, t in w.items()}
    x64 = x.detach().double().requires_grad_()
    want = _plain(w64, x64, labels, topk)
    want.backward()
    assert abs(loss.item() - want.item()) <= 3e-3 * want.item()
    for name, got, ref in [("x", x.grad, x64.grad)] + [(n, w[n].grad, w64[n].grad) for n in w]:
        off = float((got.double() - ref).norm() / ref.norm())
        assert off <= most, f"{name}: {off}"


def test_a_decoding_step_captured_and_replayed():
    """One token a sequence through norm, rotary positions, gated layer and the label loss as a scorer, replayed with a new
    token and position; the same as eager calls, bit for bit."""
    w, x, labels, _ = _weights()
    rope, norm, ffn = body.Rotary(D, layout="interleaved"), body.LayerNorm(Bt, H, train=False), body.GatedLinear(Bt, H, F, train=False)
    score = LabelLoss(Bt, H, V, train=False)
    token, at, y = x[:, 3].clone(), torch.tensor([3, 7], device="cuda"), torch.tensor([5, 9], device="cuda")

    def step():
        n = norm.forward(token, w["n1"], w["bn1"])
        q, k = rope.forward(n.view(Bt, HEADS, D), n.view(Bt, HEADS, D)[:, :KV], at)
        h = ffn.forward(n, w["gate_up"])
        out = torch.nn.functional.linear(h, w["down"])
        score.forward(out, w["head"], y)
        return q, k, h, score.losses, score.lse
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    token.copy_(x[:, 9]), at.add_(1000), y.add_(1)
    graph.replay()
    torch.cuda.synchronize()
    replayed = [t.clone() for t in outs]
    assert all(torch.equal(a, b) for a, b in zip(replayed, step()))


def _functions():
    w, x, labels, _ = _weights()
    x, flat = x.requires_grad_(), labels.reshape(-1)
    head, gu, n = (w[k].requires_grad_() for k in ("head", "gate_up", "n1"))
    rope, places = body.Rotary(D), torch.arange(S, device="cuda").expand(Bt, S)
    return {
        "layer_norm": (lambda: A.layer_norm(x, n, w["bn1"]), (x, n)),
        "rotary": (lambda: A.rotary(x.view(Bt, S, -1, D), None, places, rope), (x,)),
        "gated_linear": (lambda: A.gated_linear(x, gu), (x, gu)),
        "label_loss": (lambda: A.label_loss(x.reshape(-1, H), head, flat), (x, head)),
    }


@pytest.mark.parametrize("name", ["layer_norm", "rotary", "gated_linear", "label_loss"])
def test_second_derivatives_are_refused(name):
    f, leaves = _functions()[name]
    y = f()
    plain = torch.autograd.grad((y * y).sum(), leaves)
    y = f()
    grads = torch.autograd.grad((y * y).sum(), leaves, create_graph=True)
    assert all(torch.equal(g, p) for g, p in zip(grads, plain))
    with pytest.raises(RuntimeError, match=f"{name}.*second"):
        (sum((g.float() ** 2).sum() for g in grads) + sum((t.float() ** 2).sum() for t in leaves)).backward()


def test_what_holders_write_is_known_as_changed():
    """A graph that has saved an output of a holder says so when the holder has run again."""
    T = 24
    x, w, gu, head = (torch.randn(*s, device="cuda").to(BF16) for s in ((T, H), (H, H), (2 * F, H), (V, H)))
    y, one = torch.randint(0, V, (T,), device="cuda"), torch.ones(H, dtype=BF16, device="cuda")
    norm, ffn, ce, rope = body.LayerNorm(T, H, act8="int8", keep_y=True), body.GatedLinear(T, H, F), LabelLoss(T, H, V), body.Rotary(D)
    places, heads = torch.arange(T, device="cuda"), x.view(T, HEADS, D)
    runs = [(lambda: norm.forward(x, one, one), lambda: [norm.y]), (lambda: norm.backward(x), lambda: [norm.dx]),
            (lambda: ffn.forward(x, gu), lambda: [ffn.h]), (lambda: ffn.backward(ffn.h.clone()), lambda: [ffn.dx, ffn.dweight, ffn.dgate_up]),
            (lambda: ce.step(x, head, y), lambda: [ce.dhidden, ce.dweight, ce.loss, ce.losses]),
            (lambda: rope.forward(heads, None, places), lambda: [rope._own[0, 0]])]
    for run, outputs in runs:
        run()
        saved = [torch.mul(t, torch.ones(t.shape, dtype=t.dtype, device="cuda", requires_grad=True)) for t in outputs()]
        run()
        for g in saved:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                g.sum().backward()
    record = norm.y_record
    z = A.act8_linear(x, w.clone().requires_grad_(), record=record)
    norm.forward(x, one, one)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.sum().backward()


def test_calls_on_two_streams_at_once():
    """Holders of their own on two streams, kernels for few and for many tokens beside one another (tensor memory, clusters): the
    same bits as one after the other."""
    def calls(T, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def rand(*s):
            return torch.randn(*s, generator=g, device="cuda").to(BF16)
        h, f, v = 512, 1536, 5000
        x, gu, head, dh, one = rand(T, h), rand(2 * f, h) / 20, rand(v, h) / 20, rand(T, f), rand(h)
        y, places = torch.randint(0, v, (T,), generator=g, device="cuda"), torch.arange(T, device="cuda")
        norm, ffn, ce, rope = body.LayerNorm(T, h), body.GatedLinear(T, h, f), LabelLoss(T, h, v), body.Rotary(64)

        def run():
            out = [norm.forward(x, one, one), *norm.backward(x)]
            out += [ffn.forward(x, gu), *ffn.backward(dh)]
            out += [*ce.step(x, head, y), ce.losses, rope.forward(x.view(T, 8, 64), None, places)[0]]
            return out
        return run
    runs = [calls(T, T) for T in (1, 20, 100, 700)]
    want = [[t.clone() for t in run()] for run in runs]
    streams = [torch.cuda.Stream() for _ in runs]
    torch.cuda.synchronize()
    for _ in range(20):
        outs = []
        for run, stream in zip(runs, streams):
            with torch.cuda.stream(stream):
                outs.append(run())
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
