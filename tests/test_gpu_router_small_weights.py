"""Weights and gradients of experts far below a row's largest logit keep their digits.

The largest logit is 0, so that l - m is l itself, without a rounding, and the other
experts add less than 1e-15 to the sum, which rounds to 1.  A weight is then
scale * (exp(l) / 1): the exponential is good to 2 units in the last place (4 u;
CUDA's documentation of expf gives 1), the division by 1 and the scale, a power of
two, are exact.  With 2 u more for a factor that is a product or quotient of rounded
ones the bound is 6 u of the weight.  The exponent being rounded after a factor
log2 e, or that factor itself, would cost |l| u and more.  Backwards the gradient
of the first slot's weight alone is 1: dl_e = -p_e p_0, the bound 8 u of it for two
more products; a bf16 result has its own rounding.  (The weights, above e^-80, and
their gradients are normal numbers.)"""
import pytest
import torch

from expert_ops_util import HALF, TYPES, U, gen_of, within
from paper_2409_02227_gb300 import goldy as G

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("over", [G.GOLDY_ROUTER_ALL, G.GOLDY_ROUTER_CHOSEN])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("experts,k", [(8, 8), (64, 6), (128, 8), (256, 8), (128, 20), (300, 4), (1024, 32), (1100, 5)])
def test_far_below_the_largest(cuda_ok, experts, k, dtype, over):
    rows, gen = 200, gen_of(experts)
    l = -40 - 40 * torch.rand(rows, experts, generator=gen, device="cuda")
    l[:, 3] = 0.0
    l = l.to(TYPES[dtype][0])
    d = G.router_desc(rows, experts, k, dtype=TYPES[dtype][1], over=over, scale=0.5)
    ids = torch.empty(rows, k, dtype=torch.int32, device="cuda")
    weights, dw, dl = torch.empty(rows, k, device="cuda"), torch.zeros(rows, k, device="cuda"), torch.empty_like(l)
    dw[:, 0] = 2.0
    G.goldy_router_forward(d, l.data_ptr(), ids.data_ptr(), weights.data_ptr())
    G.goldy_router_backward(d, l.data_ptr(), ids.data_ptr(), dw.data_ptr(), dl.data_ptr())
    torch.cuda.synchronize()
    e = torch.exp(l.double())
    chosen = torch.zeros_like(e).scatter_(1, ids.long(), 1.0)
    if over == G.GOLDY_ROUTER_CHOSEN:
        e = e * chosen
    p = e / e.sum(1, keepdim=True)
    assert (ids[:, 0] == 3).all()
    want = 0.5 * p.gather(1, ids.long())
    within(weights, want, 6 * U * want, "weights")
    ref = -p * p[:, 3:4]
    ref[:, 3] = 0.0                                         # p_0 (1 - p_0), rounded
    tol = (8 * U + (HALF[torch.bfloat16] if dtype == "bf16" else 0.0)) * ref.abs()
    tol[:, 3] = 8 * U
    within(dl, ref, tol, "dlogits")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("experts", [8, 100, 256, 300, 1100])
@pytest.mark.parametrize("top", [0.0, 3e38, -2e38])
def test_logits_of_any_size(cuda_ok, experts, dtype, top):
    """Differences that overflow, and closed experts: a weight of 1, zeros, no NaN."""
    l = torch.full((9, experts), -3e38, device="cuda")
    l[:, 1::3] = -2.5e38
    l[:, 2::3] = float("-inf")
    l[:, 6] = top
    l = l.to(TYPES[dtype][0])
    d = G.router_desc(9, experts, 5, dtype=TYPES[dtype][1])
    ids = torch.empty(9, 5, dtype=torch.int32, device="cuda")
    weights, dw, dl = torch.empty(9, 5, device="cuda"), torch.ones(9, 5, device="cuda"), torch.empty_like(l)
    G.goldy_router_forward(d, l.data_ptr(), ids.data_ptr(), weights.data_ptr())
    G.goldy_router_backward(d, l.data_ptr(), ids.data_ptr(), dw.data_ptr(), dl.data_ptr())
    torch.cuda.synchronize()
    assert (ids[:, 0] == 6).all() and (ids >= 0).all()
    assert (weights[:, 0] == 1).all() and (weights[:, 1:] == 0).all() and (dl == 0).all()
