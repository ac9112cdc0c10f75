"""Tensors of the feed-forward block in any strides and at any address: the same
bits as packed copies of them give."""
import pytest
import torch

from paper_2409_02227_gb300.ffn_block import FeedForward

pytestmark = pytest.mark.gpu

ROWS, WIDTH = 100, 136


def run(x, dy, experts, ids):
    block = FeedForward(ROWS, WIDTH, 264, experts, seed=1)
    y = block.forward(x, ids)
    dx = block.backward(dy)
    torch.cuda.synchronize()
    return [y, dx] + [block.grads[k].clone() for k in sorted(block.grads)]


def odd_address(t):
    return torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)


VIEWS = {
    "transposed": lambda t: t.t().contiguous().t(),
    "columns of a wider matrix": lambda t: torch.cat([t, t], 1)[:, :WIDTH],
    "every second row": lambda t: t.repeat_interleave(2, 0)[::2],
    "one row expanded": lambda t: t[:1].expand(ROWS, WIDTH),
    "one value expanded": lambda t: t[:1, :1].expand(ROWS, WIDTH),
    "odd address": odd_address,
}


@pytest.mark.parametrize("experts", [0, 4])
@pytest.mark.parametrize("view", list(VIEWS))
def test_strides(cuda_ok, view, experts):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    x = torch.randn(ROWS, WIDTH, generator=gen, device="cuda").bfloat16()
    dy = torch.randn(ROWS, WIDTH, generator=gen, device="cuda").bfloat16()
    ids = torch.randint(0, 4, (ROWS,), generator=gen, device="cuda") if experts else None
    sx, sdy = VIEWS[view](x), VIEWS[view](dy)
    if view == "one value expanded":
        sx = x                                              # (a norm of equal values)
    for a, b in zip(run(sx, sdy, experts, ids), run(sx.clone(memory_format=torch.contiguous_format),
                                                    sdy.clone(memory_format=torch.contiguous_format), experts, ids)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.uint8, torch.int8, torch.int16, torch.int32])
def test_ids_of_any_integer_type(cuda_ok, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    x = torch.randn(ROWS, WIDTH, generator=gen, device="cuda").bfloat16()
    ids = torch.randint(0, 127, (ROWS,), generator=gen, device="cuda")
    for a, b in zip(run(x, x, 127, ids), run(x, x, 127, ids.to(dtype))):
        assert torch.equal(a, b)
