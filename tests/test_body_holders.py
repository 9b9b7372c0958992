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
