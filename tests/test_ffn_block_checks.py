"""Tensors that the feed-forward block refuses: before any CUDA call, so on the
CPU."""
import pytest
import torch

from paper_2409_02227_gb300.ffn_block import FeedForward

ROWS, WIDTH = 24, 16
GOOD = torch.zeros(ROWS, WIDTH, dtype=torch.bfloat16)
BAD = {"fewer rows": GOOD[:-1], "more rows": torch.cat([GOOD, GOOD]), "narrower": GOOD[:, :8],
       "transposed": torch.zeros(WIDTH, ROWS, dtype=torch.bfloat16), "flat": GOOD.flatten(), "fp32": GOOD.float(),
       "fp16": GOOD.half(), "one value": torch.ones((), dtype=torch.bfloat16), "another device": GOOD.to("meta")}


def block(experts=0):
    return FeedForward(ROWS, WIDTH, 32, experts, device="cpu")


@pytest.mark.parametrize("what", list(BAD))
def test_x(what):
    with pytest.raises(ValueError, match="x must be"):
        block().forward(BAD[what])
    with pytest.raises(ValueError, match="x must be"):
        block(3).forward(BAD[what], torch.zeros(ROWS, dtype=torch.int64))


@pytest.mark.parametrize("what", list(BAD))
def test_dy(what):
    b = block()
    b.x = GOOD
    with pytest.raises(ValueError, match="dy must be"):
        b.backward(BAD[what])


def test_backward_before_forward():
    with pytest.raises(RuntimeError, match="forward"):
        block().backward(GOOD)


@pytest.mark.parametrize("ids", [torch.zeros(ROWS - 1, dtype=torch.int64), torch.zeros(ROWS, 1, dtype=torch.int64),
                                 torch.zeros(ROWS), torch.zeros(ROWS, dtype=torch.bool),
                                 torch.zeros(ROWS, dtype=torch.int64, device="meta")])
def test_ids(ids):
    with pytest.raises(ValueError, match="ids must be"):
        block(3).forward(GOOD, ids)


def test_ids_and_experts_come_together():
    with pytest.raises(ValueError):
        block().forward(GOOD, torch.zeros(ROWS, dtype=torch.int64))
    with pytest.raises(ValueError):
        block(3).forward(GOOD)


def test_a_block_off_the_gpu():
    with pytest.raises(RuntimeError, match="need a GPU"):
        block().forward(GOOD)
