"""What the feed-forward block does with rows that no expert takes."""
import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from paper_2409_02227_gb300.ffn_block import FeedForward
from test_gpu_ffn_block import near, reference

pytestmark = pytest.mark.gpu


def randn(seed, *shape):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(*shape, generator=gen, device="cuda")


@pytest.mark.parametrize("strange", [-1, 5, 1 << 20])
def test_rows_without_an_expert(cuda_ok, strange):
    """Ids outside 0 .. experts - 1: the block adds nothing to such a row, its
    gradient passes through, and it reaches no parameter's gradient."""
    rows, width, hidden, experts = 300, 128, 512, 5
    # memory that the block's results are likely to get holds NaN
    junk = [torch.full((rows, w), float("nan"), device="cuda", dtype=torch.bfloat16) for w in (width, hidden) * 6]
    del junk
    block = FeedForward(rows, width, hidden, experts, seed=1)
    x, dy = randn(2, rows, width).bfloat16(), randn(3, rows, width).bfloat16()
    ids = torch.randint(0, experts, (rows,), device="cuda")
    lost = torch.zeros(rows, dtype=torch.bool, device="cuda")
    lost[::3] = True
    ids[lost] = strange
    x[0] = float("inf")                                     # not even what such a row holds
    y = block.forward(x, ids)
    dx = block.backward(dy)
    torch.cuda.synchronize()
    assert G.goldy_device_error(clear=True) == 0
    assert torch.equal(y[lost], x[lost])
    assert torch.equal(dx[lost], dy[lost])
    keep = ~lost
    ry, rdx, rg = reference(block, x[keep], ids[keep], dy[keep])
    near(y[keep], ry, "y")
    near(dx[keep], rdx, "dx")
    for k, ref in rg.items():
        near(block.grads[k], ref, k)
