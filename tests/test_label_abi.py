"""Argument checks of the label loss: found on the host before any CUDA call, so checked without a GPU (pointers are made up but
not null and aligned); and the sizes of what it needs."""
import ctypes
import math

from paper_2608_03796_b200 import binding as B
from paper_2608_03796_b200 import labels

NULL, SHAPE, ALIGN, SPACE, ARG = -1, -2, -3, -4, -5
P, Q = 0x100000, 0x200000
BIG = 1 << 40


def _call(which, **kw):
    a = labels.kdkl_label_loss_args()
    fields = dict(struct_size=ctypes.sizeof(a), label_type=1, reduction=0, dhidden_type=0, dweight_type=0, accumulate=0, temperature=1.0,
                  label_smoothing=0.1, z_loss=1e-4, ignore_index=-100, T=16, H=64, V=100, chunk=0, hidden=P, weight=P, labels=P,
                  loss=P, losses=P, lse=P, dhidden=P, dweight=P, state=Q, state_bytes=BIG, workspace=Q, workspace_bytes=BIG)
    fields.update(kw)
    for k, v in fields.items():
        setattr(a, k, v)
    return getattr(B.lib(), "kdkl_label_loss_" + which)(ctypes.byref(a), None)


def test_refusals():
    for which in ("forward", "backward", "step"):
        assert getattr(B.lib(), "kdkl_label_loss_" + which)(None, None) == NULL
        assert _call(which, struct_size=12) == ARG
        for bad in (dict(T=-1), dict(H=60), dict(H=0), dict(V=0), dict(V=1 << 31), dict(T=1 << 31)):
            assert _call(which, **bad) == SHAPE, bad
        for bad in (dict(temperature=0.0), dict(temperature=math.nan), dict(temperature=math.inf), dict(label_smoothing=-0.1),
                    dict(label_smoothing=1.1), dict(label_smoothing=math.nan), dict(z_loss=math.inf), dict(chunk=-1), dict(label_type=2), dict(reduction=2)):
            assert _call(which, **bad) == ARG, bad
        for name in ("state", "workspace", "weight", "hidden"):
            assert _call(which, **{name: None}) == NULL, name
        assert _call(which, state=Q + 16) == ALIGN and _call(which, workspace=Q + 16) == ALIGN and _call(which, hidden=P + 8) == ALIGN
        assert _call(which, weight=P + 2) == ALIGN and _call(which, token_weight=P + 2) == ALIGN and _call(which, denom_device=P + 4) == ALIGN
        assert _call(which, state_bytes=256) == SPACE and _call(which, workspace_bytes=64) == SPACE
    for which in ("forward", "step"):
        assert _call(which, loss=None) == NULL and _call(which, labels=None) == NULL and _call(which, labels=P + 4) == ALIGN
    for which in ("backward", "step"):
        assert _call(which, dhidden=None, dweight=None) == NULL and _call(which, dweight=P + 8) == ALIGN
        assert _call(which, dhidden_type=2) == ARG and _call(which, dweight_type=2) == ARG
        assert _call(which, accumulate=1) == ARG and _call(which, accumulate=2, dweight_type=1) == ARG


def test_sizes():
    """Nothing grows with T x V: the largest part is the chunk's G, 2 bytes a logit."""
    need, state = B.lib().kdkl_label_loss_workspace_bytes, B.lib().kdkl_label_loss_state_bytes
    V, H = 131072, 2048
    G = 8192 * V * 2
    one, many = need(8192, H, V, 0, 2, 0), need(262144, H, V, 0, 2, 0)
    assert G < one < 1.2 * G and many - one <= V * H * 4 + (1 << 28)        # several chunks: dweight in fp32 beside it
    assert need(262144, H, V, 0, 2, 1) < 1.2 * G and need(262144, H, V, 4096, 2, 1) < 0.6 * 1.2 * G
    assert need(262144, H, V, 0, 0, 0) < 64 << 20                           # evaluation: the partials alone
    assert state(262144) < 40 * 262144 and state(0) >= 256 and state(-1) == 0
    assert need(16, 60, 100, 0, 0, 0) == 0 and need(16, 64, 100, -1, 0, 0) == 0 and need(16, 64, 100, 0, 3, 0) == 0 and need(16, 64, 100, 0, 0, 2) == 0
