"""What a block norm keeps between its passes, and calls in the wrong order."""
import weakref

import pytest
import torch

from paper_2608_03796_b200 import body

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("args,kept", [(dict(act8="int8"), False), (dict(train=False), False), (dict(), True)])
def test_the_branch_is_kept_only_where_the_backward_pass_reads_it(args, kept):
    T, H = 8, 64
    w = torch.ones(H, dtype=BF16, device="cuda")
    join = body.BlockNorm(T, H, **args)
    b = torch.randn(T, H, device="cuda").to(BF16)
    join.forward(torch.zeros_like(b), b, w, w)
    alive = weakref.ref(b)
    del b
    assert (alive() is not None) is kept
    if args.get("train", True):
        d = join.backward(torch.ones(T, H, dtype=BF16, device="cuda"))
        assert torch.isfinite(d.branch).all()
