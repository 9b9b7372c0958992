"""One rotary table on several streams."""
import pytest
import torch

from paper_2608_03796_b200 import body

pytestmark = pytest.mark.gpu


def test_lengths_that_change_on_one_of_two_streams():
    """Each stream's outputs are its own: neither another stream's calls nor their other shapes change them, and what the
    allocator gives out meanwhile is nobody's output."""
    D, rope = 64, body.Rotary(64)
    x, n = torch.randn(500, 4, D, device="cuda"), torch.arange(500, device="cuda")
    want = rope.forward(x, None, n)[0].clone()
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    y, _ = rope.forward(x, None, n)
    for T in (500, 3, 500, 200):
        with torch.cuda.stream(other):
            z, _ = rope.forward(x[:T], None, n[:T])
        fill = [torch.full((500, 4, D), 5.0, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        assert z.data_ptr() != y.data_ptr() and torch.equal(z, want[:T]) and torch.equal(y, want)
        assert all((f == 5).all() for f in fill)
    again, _ = rope.forward(x, None, n)
    assert again.data_ptr() == y.data_ptr()


def test_captures_again_and_again():
    """What a captured call made goes with its graph: capturing the same work anew needs no more memory each time."""
    D, rope = 128, body.Rotary(128)
    x, n = torch.randn(4096, 8, D, device="cuda"), torch.arange(4096, device="cuda")
    rope.forward(x, x, n)
    torch.cuda.synchronize()
    sizes = []
    for k in range(4):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            q, key = rope.forward(x, x, n)
            total = q + key
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(total, 2 * rope.forward(x, None, n)[0])
        del graph, q, key, total
        sizes.append(torch.cuda.memory_allocated())
    assert sizes[-1] == sizes[0]


def test_frequencies_of_the_callers_own():
    """Against the rotation in 64 bits, at the tolerance of the tables that are made here (test_gpu_rotary)."""
    from tests.test_gpu_rotary import C, UNIT
    T, D, R = 200, 96, 64
    f, m = torch.rand(R // 2, dtype=torch.float64) * 3 - 1.5, 0.75
    x, n = torch.randn(T, 3, D, device="cuda"), torch.randint(-100000, 100000, (T,), device="cuda")
    y, _ = body.Rotary(D, rotary_dim=R, frequencies=f, magnitude=m).forward(x, None, n)
    angle = n.double()[:, None, None] * f.cuda()
    a, b = x[..., :R // 2].double(), x[..., R // 2:R].double()
    want = torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1) * m
    size = torch.cat([a.abs() + b.abs()] * 2, -1) * m
    assert float(((y[..., :R].double() - want).abs() - (C + 1) * UNIT * size).max()) <= 0 and torch.equal(y[..., R:], x[..., R:])
