"""Arguments that the routed feed-forward block refuses: before any CUDA call, so on
the CPU."""
import pytest
import torch

from paper_2409_02227_gb300.ffn_block import RoutedFeedForward
from test_ffn_block_checks import BAD, GOOD, ROWS, WIDTH


def block(**kw):
    return RoutedFeedForward(ROWS, WIDTH, 32, 6, 2, device="cpu", **kw)


@pytest.mark.parametrize("experts,slots", [(0, 1), (4, 0), (4, 5), (64, 33)])
def test_slots(experts, slots):
    with pytest.raises(ValueError, match="slots"):
        RoutedFeedForward(ROWS, WIDTH, 32, experts, slots, device="cpu")


@pytest.mark.parametrize("what", list(BAD))
@pytest.mark.parametrize("keep8", [False, True])
def test_tensors(what, keep8):
    with pytest.raises(ValueError, match="x must be"):
        block(keep8=keep8).forward(BAD[what])
    b = block(keep8=keep8)
    b.x = GOOD
    with pytest.raises(ValueError, match="dy must be"):
        b.backward(BAD[what])


def test_order_and_device():
    with pytest.raises(RuntimeError, match="forward"):
        block().backward(GOOD)
    with pytest.raises(RuntimeError, match="need a GPU"):
        block().forward(GOOD)
