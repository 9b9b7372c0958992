"""The device status of act8_linear's weight gradients reaches check_status, as that of the loss does."""
import pytest
import torch

from paper_2608_03796_b200 import autograd as A
from paper_2608_03796_b200 import binding as B
from paper_2608_03796_b200 import body

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _layer(seed, T=64, N=128, H=256):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(T, H, generator=g, device="cuda").to(BF16)
    w = torch.randn(N, H, generator=g, device="cuda").to(BF16).requires_grad_(True)
    return x, w


@pytest.fixture
def gives_up(monkeypatch):
    """From now on every weight gradient leaves the status of a wait that ran out (written after the kernel, which ends
    as always)."""
    run = body.Act8WeightGrad.run

    def run_and_report(self, *args, **kw):
        out = run(self, *args, **kw)
        self.workspace[:8].view(torch.int32).copy_(torch.tensor([-8, 4], dtype=torch.int32, device="cuda"))
        return out
    A.check_status()
    yield lambda: monkeypatch.setattr(body.Act8WeightGrad, "run", run_and_report)
    monkeypatch.undo()
    A.clear_cache()


def test_check_status_sees_it(gives_up):
    x, w = _layer(1)
    for _ in range(3):
        A.act8_linear(x, w).sum().backward()
    A.check_status()                                        # nothing to report
    gives_up()
    y = A.act8_linear(x, w).sum()
    y.backward()
    with pytest.raises(B.KdklError, match="act8_linear"):
        A.check_status()
    A.check_status()                                        # reported once


def test_a_later_step_sees_it(gives_up):
    x, w = _layer(2)
    gives_up()
    A.act8_linear(x, w).sum().backward()
    torch.cuda.synchronize()
    with pytest.raises(B.KdklError, match="act8_linear"):
        A.act8_linear(x, w).sum().backward()
    with pytest.raises(B.KdklError, match="act8_linear"):
        A.check_status()                                    # the later step failed as well


def test_at_once_if_asked(gives_up):
    x, w = _layer(3)
    A.act8_linear(x, w, sync_status=True).sum().backward()
    gives_up()
    with pytest.raises(B.KdklError, match="act8_linear"):
        A.act8_linear(x, w, sync_status=True).sum().backward()


def test_in_a_captured_graph(monkeypatch):
    x, w = _layer(4)
    A.act8_linear(x, w).sum().backward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    w.grad = None
    with torch.cuda.stream(side):
        A.act8_linear(x, w).sum().backward()
    torch.cuda.current_stream().wait_stream(side)
    A.check_status()
    graph = torch.cuda.CUDAGraph()
    w.grad = None
    bad = torch.tensor([-8, 4], dtype=torch.int32, device="cuda")
    run = body.Act8WeightGrad.run

    def run_and_report(self, *args, **kw):                  # nothing from the host inside a capture
        out = run(self, *args, **kw)
        self.workspace[:8].view(torch.int32).copy_(bad)
        return out
    monkeypatch.setattr(body.Act8WeightGrad, "run", run_and_report)
    with torch.cuda.graph(graph):
        A.act8_linear(x, w).sum().backward()
    monkeypatch.undo()
    graph.replay()
    with pytest.raises(B.KdklError, match="act8_linear"):
        A.check_status()
    bad.zero_()
    graph.replay()
    A.check_status()
    A.clear_cache()


def test_the_workspaces_are_not_kept():
    """What is remembered of a step is its status words: T = 6000 over one cut tile has megabytes of workspace."""
    x, w = _layer(5, T=6000, N=264, H=520)
    A.act8_linear(x, w).sum().backward()
    A.check_status()
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated()
    for _ in range(20):
        A.act8_linear(x, w).sum().backward()
    assert torch.cuda.memory_allocated() - held < 1 << 16
    A.check_status()
