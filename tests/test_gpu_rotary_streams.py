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
