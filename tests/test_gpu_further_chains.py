"""The autograd entries of the student's further operators where no other test has them: a training step that is captured and
replayed, batches without tokens, and a chunk of more than 2^31 logits."""
import pytest
import torch

from paper_2608_03796_b200 import autograd as A
from paper_2608_03796_b200 import body
from paper_2608_03796_b200.labels import LabelLoss

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
T, H, F, V, D = 200, 128, 320, 700, 32


def _leaves(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def mat(*s):
        return (torch.randn(*s, generator=g, device="cuda") / s[-1] ** 0.5).to(BF16)
    w = dict(x=mat(T, H) * H ** 0.5, gate_up=mat(2 * F, H), down=mat(H, F), head=mat(V, H), n=torch.ones(H, device="cuda").to(BF16),
             b=torch.zeros(H, device="cuda").to(BF16))
    return {k: t.requires_grad_() for k, t in w.items()}, torch.randint(0, V, (T,), generator=g, device="cuda")


def _step(w, y, rope, places, act8, single_pass):
    n = A.layer_norm(w["x"], w["n"], w["b"], **(dict(act8=act8, keep_y=True) if act8 else {}))
    n, kept = n if act8 else (n, None)
    q = A.rotary(n.view(T, -1, D), None, places, rope).reshape(T, H)
    if act8:
        h, kept = A.gated_linear(q, w["gate_up"], act8=act8, keep_h=True)
        z = A.act8_linear(h, w["down"], record=kept)
    else:
        z = torch.nn.functional.linear(A.gated_linear(q, w["gate_up"]), w["down"])
    return A.label_loss(w["x"] + z, w["head"], y, label_smoothing=0.1, single_pass=single_pass) / 3


@pytest.mark.parametrize("act8,single_pass", [(None, False), ("int8", True), ("e4m3", False)])
def test_a_training_step_captured_and_replayed(act8, single_pass):
    """The same bits as eager steps on the same values, for new values under the same graph; nothing failed on the way."""
    w, y = _leaves(0)
    rope, places = body.Rotary(D), torch.arange(T, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            for t in w.values():
                t.grad = None
            _step(w, y, rope, places, act8, single_pass).backward()
    torch.cuda.current_stream().wait_stream(side)
    for t in w.values():
        t.grad = None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = _step(w, y, rope, places, act8, single_pass)
        loss.backward()
    for seed in (1, 2):
        new, labels = _leaves(seed)
        with torch.no_grad():
            for k, t in w.items():
                t.copy_(new[k])
            y.copy_(labels), places.add_(100)
        graph.replay()
        torch.cuda.synchronize()
        A.check_status()
        want = _step(new, labels, rope, places, act8, single_pass)
        want.backward()
        A.check_status()
        assert torch.equal(loss, want)
        for k, t in w.items():
            assert torch.equal(t.grad, new[k].grad), k
    A.clear_cache()


@pytest.mark.parametrize("act8", [None, "int8"])
def test_batches_without_tokens(act8):
    """Outputs of no rows, and gradients of the weights that are zeros."""
    w, _ = _leaves(0)
    x = torch.empty(2, 0, H, dtype=BF16, device="cuda", requires_grad=True)
    places = torch.empty(2, 0, dtype=torch.int64, device="cuda")
    keep = dict(act8=act8, keep_y=True) if act8 else {}
    n = A.layer_norm(x, w["n"], w["b"], **keep)
    n, kept = n if act8 else (n, None)
    q = A.rotary(n.view(2, 0, 4, D), None, places, body.Rotary(D)).reshape(2, 0, H)
    h = A.gated_linear(q, w["gate_up"], act8=act8)
    assert h.shape == (2, 0, F)
    z = torch.nn.functional.linear(h, w["down"])
    loss = A.label_loss(z, w["head"], places) + A.label_loss(z, w["head"], places, single_pass=True) + \
        A.label_loss(z, w["head"], places, reduction="none").sum()
    loss.backward()
    A.check_status()
    assert loss.item() == 0 and x.grad.shape == x.shape
    for k in ("n", "b", "gate_up", "head"):
        assert not w[k].grad.any(), k


def test_a_chunk_of_more_than_32_bits():
    """20000 tokens x 131072 entries in one chunk, 2.6 10^9 logits, against chunks of 8192: the last rows and columns take part
    in both. dhidden's contraction goes over V in parts that depend on the rows of a chunk and is rounded once, dweight is a sum over
    tokens in fp32: both agree to the roundings of G, which are the same, and of sums of 131072 / 16 and 20000 / 16 additions."""
    many, V, H = 20000, 131072, 64
    g = torch.Generator(device="cuda").manual_seed(5)
    h = torch.randn(many, H, generator=g, device="cuda").to(BF16)
    w = (torch.randn(V, H, generator=g, device="cuda") / H ** 0.5).to(BF16)
    y = torch.randint(0, V, (many,), generator=g, device="cuda")
    y[-300:] = torch.arange(V - 300, V, device="cuda")
    kw = dict(dtype=torch.float32, dhidden_dtype=torch.float32)
    one, few = LabelLoss(many, H, V, chunk=20000, **kw), LabelLoss(many, H, V, **kw)
    for call in ("step", "backward"):
        results = []
        for op in (one, few):
            op.forward(h, w, y)
            dh, dw = op.step(h, w, y)[1:] if call == "step" else op.backward(h, w)
            assert op.status()[0] == 0
            results.append((op.losses, dh, dw))
        (la, ha, wa), (lb, hb, wb) = results
        assert torch.equal(la, lb)
        for a, b, n in ((ha, hb, V), (wa, wb, many)):
            size = float(b.abs().max())
            assert float((a - b).abs().max()) <= (n / 16 + 16) * 2.0 ** -23 * size * 4, call
