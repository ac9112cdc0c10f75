"""A feed-forward block's forward and backward pass recorded in a CUDA graph: the
replay gives the bits of the eager calls on the inputs that the buffers then hold."""
import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from paper_2409_02227_gb300.ffn_block import FeedForward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,width,hidden", [(1, 256, 512), (300, 136, 264), (40, 9000, 64)])
def test_replay(cuda_ok, rows, width, hidden):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(width)
    rnd = lambda: torch.randn(rows, width, generator=gen, device="cuda").bfloat16()  # noqa: E731
    block = FeedForward(rows, width, hidden, seed=2)
    x, dy = rnd(), rnd()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block.forward(x)
        block.backward(dy)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = block.forward(x)
        dx = block.backward(dy)
    for _ in range(3):
        x.copy_(rnd())
        dy.copy_(rnd())
        graph.replay()
        torch.cuda.synchronize()
        got = [y.clone(), dx.clone()] + [block.grads[k].clone() for k in sorted(block.grads)]
        want = [block.forward(x), block.backward(dy)] + [block.grads[k] for k in sorted(block.grads)]
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    assert G.goldy_device_error(clear=True) == 0
