"""What a rotary table owes its callers on the host. No GPU needed: the entry point is replaced where a call would reach it."""
import gc
import math
import weakref

import pytest
import torch

from paper_2608_03796_b200 import body


@pytest.fixture
def rope(monkeypatch):
    """A rotary table on the host whose calls reach nothing; (table, a function that sets the current stream, and one that says
    whether it captures)."""
    now = {"stream": 1, "capturing": False}
    monkeypatch.setattr(body, "_device", lambda: -1)
    monkeypatch.setattr(body, "_raw_stream", lambda device: now["stream"])
    monkeypatch.setattr(body, "_capturing", lambda: now["capturing"])
    r = body.Rotary(8, device="cpu")
    r._call = lambda *args: 0
    return r, lambda s: now.update(stream=s), lambda c: now.update(capturing=c)


def _turn(r, T, heads=2):
    return r.forward(torch.zeros(T, heads, 8), torch.zeros(T, 1, 8), torch.arange(T))


def test_rotary_outputs_belong_to_a_stream(rope):
    """The allocator gives freed memory to later work of the stream that it was allocated on, at once. A buffer that another
    stream's call has written, and that the next shape then replaces, would be given away under that call's kernel."""
    r, stream, _ = rope
    a = _turn(r, 3)
    stream(2)
    b = _turn(r, 3)
    assert a[0].data_ptr() != b[0].data_ptr() and a[1].data_ptr() != b[1].data_ptr()
    b = _turn(r, 5)                                                         # another length on the second stream
    stream(1)
    again = _turn(r, 3)                                                     # the first one's are where they were
    assert again[0] is a[0] and again[1] is a[1]
    assert b[0].shape == (5, 2, 8)


def test_rotary_keeps_nothing_of_a_captured_call(rope):
    """Outputs made while a graph is captured live in the graph's memory as long as the graph does; the caller has them, and a
    table that is captured again and again does not pile them up."""
    r, _, capture = rope
    eager = _turn(r, 3)
    capture(True)
    first, second = _turn(r, 3), _turn(r, 3)
    assert len({t.data_ptr() for t in (*eager, *first, *second)}) == 6
    refs = [weakref.ref(t) for t in (*first, *second)]
    del first, second
    gc.collect()
    assert all(ref() is None for ref in refs)
    capture(False)
    assert _turn(r, 3)[0] is eager[0]


def test_rotary_frequencies_of_the_callers_own():
    """Model code in wide use takes the ramp between kept and stretched frequencies linear in the pair's index, not in its turns:
    such a table, and its magnitude, go in as they are."""
    D, base, factor, length = 128, 10000.0, 16.0, 4096
    at = [D * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(base)) for turns in (32, 1)]
    low, high = max(0, math.floor(at[0])), min(D - 1, math.ceil(at[1]))
    f = base ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    keep = 1 - ((torch.arange(D // 2, dtype=torch.float64) - low) / (high - low)).clamp(0, 1)
    mine = keep * f + (1 - keep) * f / factor
    theirs = body.Rotary(D, base=base, scaling="yarn", factor=factor, original_length=length, device="cpu")
    r = body.Rotary(D, frequencies=mine, magnitude=1.25, device="cpu")
    assert torch.equal(r.turns, mine / (2 * math.pi)) and r.args.magnitude == 1.25 and r.args.turns == r.turns.data_ptr()
    assert abs(float(theirs.turns[33] / r.turns[33]) - 1) > 0.3             # the two readings differ in the middle pairs
    assert body.Rotary(D, frequencies=mine.tolist(), device="cpu").args.magnitude == 1.0
    assert body.Rotary(D, scaling="yarn", factor=factor, original_length=length, magnitude=1.0, device="cpu").args.magnitude == 1.0
    plain = body.Rotary(8, frequencies=[1.0, 0.1, 0.01, 0.001], device="cpu").turns
    assert torch.allclose(plain, body.Rotary(8, device="cpu").turns, rtol=1e-14, atol=0)
    for bad in (dict(frequencies=mine[:-1]), dict(frequencies=[math.inf] * 64), dict(frequencies=mine, scaling="linear", factor=2.0),
                dict(magnitude=math.nan), dict(magnitude=math.inf)):
        with pytest.raises(ValueError):
            body.Rotary(D, device="cpu", **bad)
