"""Which gates block_norm takes for one per channel and which for one per token, without a launch."""
import pytest
import torch

from paper_2608_03796_b200 import autograd as A


class _Taken(Exception):
    pass


@pytest.fixture(autouse=True)
def _no_launch(monkeypatch):
    def taken(residual, branch, post, pre, gate, kind, *rest):
        raise _Taken(kind)
    monkeypatch.setattr(A._BlockNorm, "apply", taken)


def _kind(branch, gate, **kw):
    x = torch.zeros(branch, dtype=torch.bfloat16)
    with pytest.raises(_Taken) as e:
        A.block_norm(x, x, gate=torch.ones(gate), **kw)
    return str(e.value)


def test_kinds():
    assert _kind((5, 8), (8,)) == "channel" and _kind((2, 5, 8), (8,)) == "channel"
    assert _kind((5, 8), (5,)) == _kind((5, 8), (5, 1)) == "token"
    assert _kind((2, 5, 8), (2, 5)) == _kind((2, 5, 8), (2, 5, 1)) == _kind((2, 5, 8), (10,)) == "token"
    assert _kind((8, 8), (8,)) == "channel" and _kind((8, 8), (8,), gate_kind="token") == "token"
    assert _kind((8, 8), (8, 1)) == "token" and _kind((1, 8, 8), (1, 8)) == "token"      # the branch's own leading shape


def test_a_row_of_channels_is_not_taken_for_tokens():
    """[1, H] broadcasts over the tokens: with as many tokens as channels it passed for one gate per token, the transposed
    gate, without an error."""
    x = torch.zeros(8, 8, dtype=torch.bfloat16)
    for shape in ((1, 8), (1, 1, 8)):
        with pytest.raises(TypeError, match="one per channel"):
            A.block_norm(x, x, gate=torch.ones(shape))
    assert _kind((8, 8), (1, 8), gate_kind="channel") == "channel"
