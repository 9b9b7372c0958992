"""What a call writes is known to autograd as changed: a graph that has saved it says so instead of using the new values."""
import pytest
import torch

from paper_2608_03796_b200 import autograd as A
from paper_2608_03796_b200 import body

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
T, H, N = 40, 64, 96


def _randn(seed, *shape, dtype=BF16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def _refused(y):
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_a_record_written_again_before_the_backward_pass():
    x, w = _randn(1, T, H), _randn(2, N, H).requires_grad_(True)
    rec = body.Act8Record(T, H).store(x)
    y = A.act8_linear(x, w, record=rec)
    y.sum().backward()                                      # nobody has touched it
    y = A.act8_linear(x, w, record=rec)
    rec.store(2 * x)
    _refused(y)


def test_records_of_holders_that_ran_again():
    x, w, one = _randn(1, T, H), _randn(2, N, H).requires_grad_(True), torch.ones(H, dtype=BF16, device="cuda")
    join, ffn = body.BlockNorm(T, H, act8="int8", keep_y=True), body.GatedAct(T, H, keep_h=True)
    for run, records in ((lambda: join.forward(x, x, one, one), lambda: (join.y_record, join.branch_record, join.sum_record)),
                         (lambda: ffn.forward(x, x), lambda: (ffn.h_record, ffn.gate_record, ffn.up_record))):
        run()
        ys = [A.act8_linear(x, w, record=r) for r in records()]
        run()
        for y in ys:
            _refused(y)


def test_outputs_that_a_graph_has_saved():
    x, dy, one = _randn(1, T, H), _randn(3, T, N), torch.ones(H, dtype=BF16, device="cuda")
    w = _randn(2, H, H).requires_grad_(True)
    rec = body.Act8Record(T, H).store(x)
    out = torch.empty(T, H, dtype=BF16, device="cuda")
    join, ffn, grad = body.BlockNorm(T, H, gate="channel"), body.GatedAct(T, H), body.Act8WeightGrad(T, N, H)
    runs = [(lambda: rec.load(out), lambda: [out]),
            (lambda: join.forward(x, x, one, one, one), lambda: [join.y, join.sum]),
            (lambda: join.backward(x, x), lambda: [join.dresidual, join.dbranch]),
            (lambda: ffn.forward(x, x), lambda: [ffn.h]),
            (lambda: ffn.backward(x), lambda: list(ffn.halves)),
            (lambda: grad.run(dy, rec), lambda: [grad.dweight])]
    for run, outputs in runs:
        run()
        ys = [torch.nn.functional.linear(t, w) for t in outputs()]          # saves t for w's gradient
        run()
        for y in ys:
            _refused(y)
    d = join.backward(x, x)
    p = torch.ones(H, dtype=BF16, device="cuda", requires_grad=True)
    ys = [t * p for t in (d.post_weight, d.pre_weight, d.gate)]
    join.backward(x, x)
    for y in ys:
        _refused(y)
    total = torch.zeros(N, H, dtype=BF16, device="cuda")
    y = torch.nn.functional.linear(total, w)
    grad.run(dy, rec, out=total, accumulate=True)
    _refused(y)


def test_holders_made_in_inference_mode_still_run():
    x = _randn(1, T, H)
    with torch.inference_mode():
        rec = body.Act8Record(T, H)
        ffn = body.GatedAct(T, H)
    want = body.Act8Record(T, H).store(x).load()
    assert torch.equal(rec.store(x).load(), want)
    with torch.inference_mode():
        assert torch.equal(rec.store(x).load(), want)
        ffn.forward(x, x)
    ffn.forward(x, x)
