"""Every row of a router's batch by itself: the ids, weights and gradient of a row
have the same bits alone, at any place of a batch and beside any other rows; equal
logits of a row are chosen in the order of their indices and weigh the same."""
import math

import pytest
import torch

from expert_ops_util import TYPES, gen_of
from paper_2409_02227_gb300 import goldy as G
from test_gpu_router import choose

pytestmark = pytest.mark.gpu
ALL, CHOSEN = G.GOLDY_ROUTER_ALL, G.GOLDY_ROUTER_CHOSEN


def run(l, dw, k, dtype, over):
    """(ids, weights, dlogits) of the rows of `l`, packed."""
    rows, experts = l.shape
    d = G.router_desc(rows, experts, k, dtype=TYPES[dtype][1], over=over, scale=1.25)
    l, dw = l.contiguous(), dw.contiguous()
    ids = torch.full((rows, k), 12345, dtype=torch.int32, device="cuda")
    weights, dl = torch.full((rows, k), math.nan, device="cuda"), torch.full_like(l, math.nan)
    G.goldy_router_forward(d, l.data_ptr(), ids.data_ptr(), weights.data_ptr())
    G.goldy_router_backward(d, l.data_ptr(), ids.data_ptr(), dw.data_ptr(), dl.data_ptr())
    torch.cuda.synchronize()
    return ids, weights, dl


def same(got, want):
    assert torch.equal(got[0], want[0])
    for g, w in zip(got[1:], want[1:]):
        whole = torch.int32 if g.dtype == torch.float32 else torch.int16
        assert torch.equal(g.view(whole), w.view(whole))


@pytest.mark.parametrize("over", [ALL, CHOSEN])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("experts,k", [(5, 3), (64, 6), (100, 7), (128, 8), (256, 8), (128, 20), (300, 4), (1100, 5)])
def test_alone_and_in_a_batch(cuda_ok, experts, k, dtype, over):
    """Untied rows with tied, closed and infinite ones between them."""
    rows, gen = 41, gen_of(experts + k)
    l = torch.randn(rows, experts, generator=gen, device="cuda") * 3
    dw = torch.randn(rows, k, generator=gen, device="cuda")
    l[3::4] = l[3::4].round()                               # ties in every fourth row
    l[9] = 0.5
    l[13, k // 2:] = -math.inf                              # fewer open experts than slots
    l[17] = -math.inf
    l[21, :2] = math.nan
    l[25, 1] = math.inf
    l = l.to(TYPES[dtype][0])
    whole = run(l, dw, k, dtype, over)
    for r in range(rows):
        same(run(l[r:r + 1], dw[r:r + 1], k, dtype, over), [t[r:r + 1] for t in whole])
    order = torch.randperm(rows, generator=gen, device="cuda")
    same(run(l[order], dw[order], k, dtype, over), [t[order] for t in whole])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("levels", [1, 2, 7, 40])
@pytest.mark.parametrize("experts", [8, 31, 64, 128, 200, 256])
def test_few_different_values(cuda_ok, experts, levels, dtype):
    """Ties among the chosen logits and for the last slot, any number of slots."""
    rows, gen = 70, gen_of(experts + levels)
    l = torch.randint(0, levels, (rows, experts), generator=gen, device="cuda") * 0.25 - 1.0
    l = torch.where((l == 0) & (torch.rand(rows, experts, generator=gen, device="cuda") < 0.5), -0.0, l)
    l[torch.rand(rows, experts, generator=gen, device="cuda") < 0.2] = -math.inf
    l = l.to(TYPES[dtype][0])
    for k in range(1, 9):
        ids, weights, _ = run(l, torch.zeros(rows, k, device="cuda"), k, dtype, ALL)
        want = choose(l, k)
        assert torch.equal(ids.long(), want)
        v = torch.where(want < 0, -math.inf, l.double().gather(1, want.clamp(min=0)))
        equal = v[:, 1:] == v[:, :-1]
        assert torch.equal(weights[:, 1:][equal], weights[:, :-1][equal])
        assert (weights[:, 1:] <= weights[:, :-1]).all() and (weights[want < 0] == 0).all()


@pytest.mark.parametrize("experts,k", [(20, 4), (128, 8), (256, 5)])
def test_several_nan(cuda_ok, experts, k):
    """NaNs come first, in the order of their indices, then infinities in theirs."""
    l = torch.randn(9, experts, generator=gen_of(2), device="cuda")
    l[4, 17], l[4, 3] = math.nan, math.nan
    l[4, 11], l[4, 2] = math.inf, math.inf
    ids, weights, _ = run(l, torch.zeros(9, k, device="cuda"), k, "f32", ALL)
    assert ids[4, :4].tolist() == [3, 17, 2, 11]
    rest = [r for r in range(9) if r != 4]
    assert torch.equal(ids[rest].long(), choose(l[rest], k)) and torch.isfinite(weights[rest]).all()
