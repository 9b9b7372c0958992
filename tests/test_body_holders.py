"""What the holders of the student-body operators owe their callers on the host: refusals, and what they keep. No GPU needed:
entry points are replaced where a call would reach them."""
import pytest
import torch

from paper_2608_03796_b200 import body

P = 0x100000


def test_holders_on_another_device_are_refused_before_a_launch(monkeypatch):
    """Records, workspaces and outputs travel to the kernels as stored addresses: a holder whose memory is on the host or
    on another GPU than the current one is refused by every call. The arguments are taken as good here, the current
    device as cuda:0, and no entry point may be reached."""
    T, H = 4, 64
    monkeypatch.setattr(body, "_rows", lambda t, T, H, dtype, name: (P, H))
    monkeypatch.setattr(body, "_vector", lambda t, n, dtype, name: P)
    monkeypatch.setattr(body, "_device", lambda: 0)
    monkeypatch.setattr(body, "_raw_stream", lambda device: 0)

    def reached(*args):
        raise AssertionError("an address of another device reached the library")
    x = torch.zeros(T, H, dtype=torch.bfloat16)
    w = torch.ones(H, dtype=torch.bfloat16)

    def holders():
        rec = body.Act8Record(T, H, device="cpu")
        held = body.Act8Record(T, H, buffer=torch.zeros(rec.nbytes, dtype=torch.uint8))
        grad = body.Act8WeightGrad(T, 8, H, device="cpu")
        ffn, join = body.GatedAct(T, H, device="cpu"), body.BlockNorm(T, H, act8="int8", device="cpu")
        plain = body.BlockNorm(T, H, device="cpu")
        for r in (rec, held):
            r._store = r._load = reached
        grad._run = ffn._forward = ffn._backward = join._forward = join._backward = reached
        plain._forward = plain._backward = reached
        ffn.stored = True
        join.kept = plain.kept = (x, x, w, w, None)
        return rec, held, grad, ffn, join, plain
    rec, held, grad, ffn, join, plain = holders()
    here = body.Act8Record(T, H, device="cpu")
    here.at = 0                                                             # as if it were on the current device
    for call in (lambda: rec.store(x), lambda: rec.load(x), lambda: held.store(x), lambda: held.load(x),
                 lambda: grad.run(x, rec), lambda: grad.run(x, here), lambda: ffn.forward(x, x), lambda: ffn.backward(x),
                 lambda: join.forward(x, x, w, w), lambda: join.backward(x, x),
                 lambda: plain.forward(x, x, w, w), lambda: plain.backward(x, x)):
        with pytest.raises(TypeError, match="on the host"):
            call()
    rec, held, grad, ffn, join, plain = holders()
    for h in (rec, held, grad, ffn, join, plain):
        h.at = 1
    for call in (lambda: rec.store(x), lambda: grad.run(x, rec), lambda: ffn.forward(x, x), lambda: plain.forward(x, x, w, w)):
        with pytest.raises(TypeError, match="cuda:1"):
            call()
    grad.at, ffn.at, join.at = 0, 0, 0                                      # the holder is here, a record of it is not
    for call in (lambda: grad.run(x, rec), lambda: ffn.backward(x), lambda: join.backward(x, x)):
        with pytest.raises(TypeError, match="record"):
            call()


def test_what_a_call_writes_is_marked_as_changed(monkeypatch):
    """Autograd's version counters, by which a graph knows that a tensor it has saved was changed, without a launch."""
    T, H, N = 4, 64, 8
    monkeypatch.setattr(body, "_rows", lambda t, T, H, dtype, name: (P, H))
    monkeypatch.setattr(body, "_vector", lambda t, n, dtype, name: P)
    monkeypatch.setattr(body, "_stream", lambda at, what: 0)
    x, w = torch.zeros(T, H, dtype=torch.bfloat16), torch.ones(H, dtype=torch.bfloat16)
    rec = body.Act8Record(T, H, device="cpu")
    grad = body.Act8WeightGrad(T, N, H, device="cpu")
    ffn = body.GatedAct(T, H, device="cpu", keep_h=True)
    join = body.BlockNorm(T, H, act8="int8", gate="channel", keep_y=True, device="cpu")
    rec._store = rec._load = grad._run = ffn._forward = ffn._backward = join._forward = join._backward = lambda *args: 0
    out, dy = torch.empty(T, H, dtype=torch.bfloat16), torch.zeros(T, N, dtype=torch.bfloat16)
    ffn.forward(x, x), ffn.backward(x), join.forward(x, x, w, w, w), join.backward(x, x)
    for call, written in ((lambda: rec.store(x), [rec.buffer]), (lambda: rec.load(out), [out]),
                          (lambda: grad.run(dy, rec), [grad.dweight]),
                          (lambda: ffn.forward(x, x), [ffn.h, ffn.gate_record.buffer, ffn.up_record.buffer, ffn.h_record.buffer]),
                          (lambda: ffn.backward(x), [ffn.dgate_up, *ffn.halves]),
                          (lambda: join.forward(x, x, w, w, w), [join.y, join.sum, join.branch_record.buffer,
                                                                 join.sum_record.buffer, join.y_record.buffer]),
                          (lambda: join.backward(x, x), [join.dresidual, join.dbranch, *join.grads.values()])):
        before = [t._version for t in written]
        call()
        assert all(t._version > v for t, v in zip(written, before))
    assert x._version == w._version == 0                                    # inputs are not


def test_a_block_norms_backward_call_before_any_forward_call():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    for act8 in (None, "int8"):
        with pytest.raises(RuntimeError, match="before any forward"):
            body.BlockNorm(4, 64, act8=act8, device="cpu").backward(x, x)


def test_a_gated_activations_backward_call_before_any_forward_call():
    """Its records hold nothing yet."""
    with pytest.raises(RuntimeError, match="before any forward"):
        body.GatedAct(4, 64, device="cpu").backward(torch.zeros(4, 64, dtype=torch.bfloat16))


def test_a_record_of_y_needs_a_y():
    """Without a pre norm there is no y: its record would go on holding the call's before, or nothing."""
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.ones(64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="keep_y"):
        body.BlockNorm(4, 64, act8="int8", keep_y=True, device="cpu").forward(x, x, post_weight=w)
