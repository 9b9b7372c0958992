"""What the label loss's holder keeps. No GPU needed: entry points are replaced where a call would reach them."""
import pytest
import torch

from paper_2608_03796_b200 import labels

BF16, F32 = torch.bfloat16, torch.float32
P = 0x100000


def _label(monkeypatch, **kw):
    monkeypatch.setattr(labels, "_rows", lambda t, T, H, dtype, name: (P, H))
    monkeypatch.setattr(labels, "_vector", lambda t, n, dtype, name: P)
    monkeypatch.setattr(labels, "_stream", lambda at, what: 0)
    op = labels.LabelLoss(300, 64, 5000, device="cpu", **kw)
    given = []
    op._calls = tuple(lambda ref, stream: given.append((op.args.workspace, op.args.workspace_bytes)) or 0 for _ in range(3))
    return op, given


@pytest.mark.parametrize("order", ["backward first", "step first"])
def test_label_loss_has_one_workspace_for_gradients(monkeypatch, order):
    """The part of two bytes a logit is scratch: backward and step calls share it, and it is never replaced (a captured graph may
    hold its address)."""
    op, given = _label(monkeypatch)
    h, w, y = torch.zeros(300, 64, dtype=BF16), torch.zeros(5000, 64, dtype=BF16), torch.zeros(300, dtype=torch.int64)
    op.forward(h, w, y)
    small = given[0][1]
    for call in (("backward", "step", "backward") if order == "backward first" else ("step", "backward", "step")):
        op.backward(h, w) if call == "backward" else op.step(h, w, y)
    grads = set(given[1:])
    assert len(grads) == 1 and grads.pop()[1] == max(op._need(1), op._need(2)) and small == op._need(0) < op._need(2)
    op.forward(h, w, y)
    assert sum(t.numel() for t in op.workspaces.values()) <= small + max(op._need(1), op._need(2))


def test_label_loss_fills_nothing_that_a_call_overwrites(monkeypatch):
    """dweight is written whole, or added to: only a sum of the holder's own starts from zeros."""
    op, _ = _label(monkeypatch, dtype=F32)
    zeros, made = torch.zeros, []
    monkeypatch.setattr(labels.torch, "zeros", lambda *a, **kw: made.append(a) or zeros(*a, **kw))
    op._outputs(None, False)
    assert not made and op.dweight.shape == (5000, 64)
    op, _ = _label(monkeypatch, dtype=F32)
    made.clear()
    op._outputs(None, True)
    assert made[-1][:2] == (5000, 64) and not op.dweight.any()
