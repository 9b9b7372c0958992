"""Chains of student-body calls without a wait of the host in between: every kernel of them may start while the one
before it still runs, and reads what that one wrote, over buffers that the call before last has used as well.
Results are compared bit for bit with the same calls made one at a time on buffers of their own."""
import pytest
import torch

from paper_2608_03796_b200 import body

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _randn(seed, *shape, dtype=BF16, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


# one tile; several tiles, none of them cut; tiles that are cut into parts; the form for rows that are not whole words
@pytest.mark.parametrize("T,N,H", [(40, 64, 96), (300, 512, 768), (2500, 1000, 1544), (40, 33, 65)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_accumulating_into_one_buffer(T, N, H, dtype):
    """out = round(out + dW_k) for each k: the fp32 sum of a call that does not accumulate, plus the old value, rounded
    once to the output's type."""
    K = 12
    rec = body.Act8Record(T, H).store(_randn(1, T, H))
    dys = [_randn(10 + k, T, N) for k in range(K)]
    one = body.Act8WeightGrad(T, N, H, dtype=F32)
    parts = []
    for dy in dys:
        parts.append(one.run(dy, rec).clone())
        torch.cuda.synchronize()
    start = _randn(2, N, H, dtype=dtype)
    want = start.clone()
    for p in parts:
        want = (want.float() + p).to(dtype)
    op = body.Act8WeightGrad(T, N, H, dtype=dtype)
    for _ in range(4):
        out = start.clone()
        for dy in dys:
            op.run(dy, rec, out=out, accumulate=True)
        assert torch.equal(out, want)


@pytest.mark.parametrize("T,H", [(1, 64), (7, 264), (33, 1001), (300, 4096)])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_one_record_used_again_and_again(T, H, fmt):
    xs = [_randn(k, T, H, dtype=(BF16, F32, torch.float16)[k % 3], scale=2.0 ** (k % 5)) for k in range(16)]
    want = []
    for x in xs:
        want.append(body.Act8Record(T, H, fmt).store(x).load(dtype=F32))
        torch.cuda.synchronize()
    rec = body.Act8Record(T, H, fmt)
    outs = [torch.empty(T, H, dtype=F32, device="cuda") for _ in xs]
    for _ in range(4):
        for x, out in zip(xs, outs):
            rec.store(x).load(out)
        for out, w in zip(outs, want):
            assert torch.equal(out, w)
            out.zero_()


@pytest.mark.parametrize("T,H", [(1, 64), (7, 264), (33, 1001), (300, 1024), (5, 16384)])
@pytest.mark.parametrize("fmt", ["int8", None])
def test_one_join_and_one_gated_activation_used_again_and_again(T, H, fmt):
    """Forward and backward of both over one set of buffers, inputs, weights and gates changing from step to step; the
    join's outputs are the gated activation's inputs, and its sum is the next step's residual."""
    steps = 8
    data = [dict(b=_randn(100 + k, T, H), dy=_randn(200 + k, T, H), dx=_randn(300 + k, T, H),
                 w=1 + _randn(400 + k, H, scale=0.1), g=_randn(500 + k, T, scale=0.5)) for k in range(steps)]

    def holders():
        return (body.BlockNorm(T, H, gate="token", act8=fmt, keep_y=fmt is not None), body.GatedAct(T, H, act8=fmt))

    def step(join, ffn, r, d, wait):
        y, x = join.forward(r, d["b"], d["w"], d["w"], d["g"])
        h = ffn.forward(y, x)
        if wait:
            torch.cuda.synchronize()
        outs = [y, x, h, *join.backward(d["dy"], d["dx"])]
        if fmt is not None:
            outs += [*ffn.backward(d["dy"]), join.y_record.load(dtype=F32)]
        return outs
    first, want = _randn(9, T, H), []
    r = first
    for d in data:
        outs = step(*holders(), r, d, True)
        torch.cuda.synchronize()
        want.append(outs)
        r = outs[1]
    pair = [holders(), holders()]                       # a step's residual is the other holder's sum, not its own output
    for _ in range(3):
        r, got = first, []
        for k, d in enumerate(data):
            outs = step(*pair[k % 2], r, d, False)
            r = outs[1]
            # a copy starts only when the kernels before it have ended, so most steps are without
            got.append([t.clone() for t in outs] if k % 3 == 2 or k >= steps - 2 else None)
        for outs, w in zip(got, want):
            assert outs is None or all(torch.equal(a, c) for a, c in zip(outs, w))
