"""Device statuses that are still to be looked at, without a GPU: the words are put where a finished copy leaves them."""
import pytest
import torch

from paper_2608_03796_b200 import autograd as A
from paper_2608_03796_b200 import binding as B


class _Ended:
    waited = 0

    def synchronize(self):
        self.waited += 1

    def query(self):
        return True


def _pending(code, where, what="act8_linear"):
    op = A._StepStatus()
    op.what, op.probe_pending, op.probe_event = what, True, _Ended()
    op.probe = torch.tensor([code, where, 0, 0], dtype=torch.int32)
    A._probed.append(op)
    return op


def test_every_pending_step_is_looked_at_and_the_first_failure_raised():
    ops = [_pending(0, 0), _pending(-8, 4), _pending(-8, 7), _pending(0, 0)]
    with pytest.raises(B.KdklError, match="act8_linear step, detail 4"):
        A.check_status()
    assert not A._probed and all(op.probe_event.waited == 1 for op in ops) and all(op in A._idle for op in ops)
    A.check_status()
    A._idle.clear()


def test_a_step_of_a_captured_graph():
    A._captured.append(("act8_linear", torch.tensor([0, 0, 0, 0], dtype=torch.int32)))
    A.check_status()
    A._captured[0][1][0] = -8
    with pytest.raises(B.KdklError, match="captured act8_linear"):
        A.check_status()
    with pytest.raises(B.KdklError):
        A.clear_cache()
    assert not A._captured
