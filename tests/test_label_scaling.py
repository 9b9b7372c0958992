"""Argument checks of kdkl_label_loss_rescale: found on the host before any CUDA call (pointers are made up but aligned)."""
from paper_2608_03796_b200 import binding as B

P = 0x100000


def test_refusals():
    call = B.lib().kdkl_label_loss_rescale
    assert call(P, 2, 8, P, P, None) == -5 and call(P, -1, 8, P, P, None) == -5
    for count in (-8, 4, 12, 1 << 60):
        assert call(P, 0, count, P, P, None) == -2
    assert call(None, 0, 8, P, P, None) == -1 and call(P, 0, 8, None, P, None) == -1 and call(P, 0, 8, P, None, None) == -1
    assert call(P + 8, 0, 8, P, P, None) == -3 and call(P, 1, 8, P, P + 4, None) == -3 and call(P, 0, 8, P + 2, P, None) == -3
    assert call(None, 0, 0, P, None, None) == 0
