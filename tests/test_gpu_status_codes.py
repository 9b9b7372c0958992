"""What a status block holds when more than one thing happens: entries that were ignored (KDKL_ERR_INDEX, the results stand) must
not hide an error that comes after them."""
import pytest
import torch

from paper_2608_03796_b200 import binding as B
from paper_2608_03796_b200.labels import LabelLoss

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _label_inputs(T, H, V):
    g = torch.Generator(device="cuda").manual_seed(T)
    h = torch.randn(T, H, generator=g, device="cuda").to(BF16)
    w = (torch.randn(V, H, generator=g, device="cuda") / H ** 0.5).to(BF16)
    return h, w, torch.randint(0, V, (T,), generator=g, device="cuda")


@pytest.mark.parametrize("before,after", [((0, 0), (-8, 99)), ((-10, 0), (-8, 99)), ((-11, 5), (-11, 5)), ((-9, 0), (-9, 0))])
def test_a_wait_that_runs_out(before, after):
    """The first error stays; a note does not stand in its way."""
    words = torch.tensor(before, dtype=torch.int32, device="cuda")
    B.kdkl_wait_selftest(words, 50_000_000)
    assert tuple(words.tolist()) == after


def test_a_state_of_another_call_behind_a_label_out_of_range():
    T, H, V = 600, 64, 200
    h, w, y = _label_inputs(T, H, V)
    y[3] = V
    op = LabelLoss(T, H, V)
    op.forward(h, w, y)
    assert op.status()[0] == -10
    other = LabelLoss(T, H, V, chunk=256)
    other.fed = True
    other.state.copy_(op.state)
    other._outputs(None, False)
    other.dhidden.fill_(7), other.dweight.fill_(7)
    dh, dw = other.backward(h, w)
    code, detail = other.status()
    assert code == -9 and detail[2] == 1 and (dh == 7).all() and (dw == 7).all()


def test_a_label_out_of_range_alone():
    """Through all calls it stays what is reported, with its count."""
    T, H, V = 300, 64, 200
    h, w, y = _label_inputs(T, H, V)
    y[3] = y[70] = V
    op = LabelLoss(T, H, V)
    op.forward(h, w, y), op.backward(h, w)
    assert op.status()[0] == -10 and op.status()[1][2] == 2
    op.step(h, w, y)
    assert op.status()[0] == -10 and op.status()[1][2] == 2


def test_a_loss_that_is_not_finite_behind_an_index_out_of_range():
    """The loss against a teacher notes the index in its first kernel, before there is any loss."""
    T, H, V, K = 300, 64, 200, 4
    h, w, _ = _label_inputs(T, H, V)
    idx = torch.stack([torch.randperm(V, device="cuda")[:K] for _ in range(T)]).int()
    val = torch.randn(T, K, device="cuda")
    idx[7, 1] = V
    op = B.FusedChunkedKL(T, H, V, K)
    op.forward(h, w, idx, val)
    assert op.status()[0] == -10
    h[9] = float("inf")
    op.forward(h, w, idx, val)
    code, detail = op.status()
    assert code == -11 and detail[0] == 9 and detail[2] == 1
