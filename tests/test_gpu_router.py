"""The router against its definition in fp64.

Bounds.  A weight is scale e_j / sum(e), e = exp(l - m) = 2^((l - m) log2 e): the
difference, the constant and their product are rounded, 2.3 |l - m| u of e
together, and the power is good to 2 units in the last place (4 u).  In the sum
that is 2.3 sum(p |l - m|) u, and sum(p |l - m|) is at most ln(experts) < 8.4, so 20
u; the sum has experts / 8 + 5 steps, the division and the scale one rounding each:
with logits that spread over `spread`, (2.3 spread + experts / 8 + 36) u of the weight.
dl_e = p_e (g_e - sum g p): p as above, the dot product over at most k terms has 6
steps more, so twice that bound of p_e (|g_e| + sum |g| p), then one rounding to
the logits' type."""
import math

import pytest
import torch

from expert_ops_util import HALF, TYPES, U, Rows, gen_of, within
from paper_2409_02227_gb300 import goldy as G

pytestmark = pytest.mark.gpu
ALL, CHOSEN = G.GOLDY_ROUTER_ALL, G.GOLDY_ROUTER_CHOSEN


def choose(l, k):
    """The k largest, ties to the lowest index; -1 where none but closed ones are left."""
    left, ids = l.double().clone(), []
    index = torch.arange(l.shape[1], device=l.device)
    for _ in range(k):
        best = left.max(1, keepdim=True).values
        at = torch.where(left == best, index, l.shape[1]).min(1).values
        ids.append(torch.where(best[:, 0] == -math.inf, -1, at))
        left.scatter_(1, at[:, None], -math.inf)
    return torch.stack(ids, 1)


def softmax(l, ids, over):
    l = l.double()
    if over == CHOSEN:
        one = torch.zeros(l.shape[0], l.shape[1] + 1, device=l.device).scatter_(1, torch.where(ids < 0, l.shape[1], ids), 1.0)
        l = torch.where(one[:, :-1] > 0, l, -math.inf)
    m = l.max(1, keepdim=True).values
    e = torch.exp(l - torch.where(m == -math.inf, 0.0, m))
    return e / e.sum(1, keepdim=True).clamp(min=1e-300)


def at(t, ids):
    return torch.where(ids < 0, 0.0, t.gather(1, ids.clamp(min=0)))


def check(l, rows, experts, k, over, dtype, scale, forward, seed=0, dw=None, ids=None):
    """Both calls on the logits in `l`; returns (ids, weights, dlogits)."""
    d = G.router_desc(rows, experts, k, dtype=TYPES[dtype][1], over=over, scale=scale, ld=l.ld, ldd=experts + 3)
    out_ids = torch.full((rows, k), 12345, dtype=torch.int32, device="cuda")
    weights = torch.full((rows, k), math.nan, device="cuda")
    G.goldy_router_forward(d, l.ptr, out_ids.data_ptr(), weights.data_ptr())
    dw = torch.randn(rows, k, generator=gen_of(seed), device="cuda") if dw is None else dw
    dl = Rows(rows, experts, TYPES[dtype][0], experts + 3, 1)
    used = out_ids if ids is None else ids
    G.goldy_router_backward(d, l.ptr, used.data_ptr(), dw.data_ptr(), dl.ptr)
    torch.cuda.synchronize()
    assert l.guarded() and dl.guarded()
    return out_ids, weights, dl.t, dw


def against_fp64(l, k, over, dtype, scale, ids, weights, dl, dw, forward_ids=None):
    rows, experts = l.shape
    finite = torch.where(torch.isfinite(l.double()), l.double(), 0.0)
    spread = float((finite.max(1).values - finite.min(1).values).max()) if rows else 0.0
    eps = (2.3 * spread + experts / 8 + 36) * U
    want = choose(l, k)
    if forward_ids is None:
        assert torch.equal(ids.long(), want)
        p = softmax(l, want, over)
        w = abs(scale) * at(p, want)
        within(weights, scale * at(p, want), eps * w, "weights")
        used = want
    else:
        used = torch.where((forward_ids < 0) | (forward_ids >= experts), -1, forward_ids).long()
        p = softmax(l, used, over)
    spare = torch.where(used < 0, experts, used)
    g = torch.zeros(rows, experts + 1, dtype=torch.float64, device="cuda").scatter_add_(1, spare, scale * dw.double())[:, :-1]
    ga = torch.zeros(rows, experts + 1, dtype=torch.float64, device="cuda").scatter_add_(1, spare, (scale * dw.double()).abs())[:, :-1]
    ref = p * (g - (g * p).sum(1, keepdim=True))
    size = p * (ga + (ga * p).sum(1, keepdim=True))
    # a bf16 result below the smallest normal number is off by half of a fixed step
    within(dl, ref, HALF[TYPES[dtype][0]] * ref.abs() + 2 * eps * size + 1e-38, "dlogits")


@pytest.mark.parametrize("over", [ALL, CHOSEN])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,experts,k", [(1, 1, 1), (3, 2, 2), (5, 31, 8), (64, 32, 32), (9, 33, 3), (200, 60, 6),
                                            (1000, 64, 8), (77, 100, 7), (40, 128, 1), (1300, 256, 8), (33, 257, 16),
                                            (17, 512, 4), (9, 1000, 5), (6, 1024, 32), (5, 1025, 8), (4, 4096, 32)])
def test_sizes(cuda_ok, rows, experts, k, dtype, over):
    gen = gen_of(rows + experts)
    l = Rows(rows, experts, TYPES[dtype][0], experts + (experts % 3), experts % 2,
             2.0 * torch.randn(rows, experts, generator=gen, device="cuda"))
    ids, weights, dl, dw = check(l, rows, experts, k, over, dtype, 1.5, True)
    against_fp64(l.t, k, over, dtype, 1.5, ids, weights, dl, dw)


@pytest.mark.parametrize("over", [ALL, CHOSEN])
@pytest.mark.parametrize("experts,k", [(8, 3), (64, 6), (200, 8), (2000, 5)])
def test_closed_experts_and_rows(cuda_ok, experts, k, over):
    """Closed experts are never chosen; rows with fewer open ones than slots, and with none."""
    rows, gen = 60, gen_of(3)
    v = torch.randn(rows, experts, generator=gen, device="cuda")
    for r in range(rows):                                   # r open experts, then all of them
        if r < 30:
            v[r, torch.randperm(experts, generator=gen, device="cuda")[min(r % (k + 3), experts):]] = -math.inf
    l = Rows(rows, experts, torch.float32, fill=v)
    ids, weights, dl, dw = check(l, rows, experts, k, over, "f32", 1.0, True)
    against_fp64(l.t, k, over, "f32", 1.0, ids, weights, dl, dw)
    assert (ids[0] == -1).all() and (weights[0] == 0).all() and (dl[0] == 0).all()
    assert (dl[torch.isinf(v)] == 0).all()


@pytest.mark.parametrize("experts,k", [(7, 4), (64, 8), (130, 32), (1500, 9)])
def test_ties(cuda_ok, experts, k):
    """Few different values, 0 and -0 among them: the lowest index first."""
    rows, gen = 50, gen_of(4)
    v = torch.randint(-1, 2, (rows, experts), generator=gen, device="cuda").float()
    v = torch.where((v == 0) & (torch.rand(rows, experts, generator=gen, device="cuda") < 0.5), -0.0, v)
    v[0] = -0.0
    v[1] = -math.inf
    for dtype in ("bf16", "f32"):
        l = Rows(rows, experts, TYPES[dtype][0], fill=v)
        ids, weights, dl, dw = check(l, rows, experts, k, ALL, dtype, 1.0, True)
        against_fp64(l.t, k, ALL, dtype, 1.0, ids, weights, dl, dw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("experts", [20, 300, 1300])
def test_infinite_and_nan(cuda_ok, experts, dtype):
    """A NaN or +infinity is chosen first; its row's weights are NaN, others' are not."""
    v = torch.randn(6, experts, generator=gen_of(5), device="cuda")
    v[1, 13], v[1, 4] = math.nan, math.inf
    v[2, 9] = math.inf
    v.view(torch.int32)[3, 2] = -1                          # a NaN with its sign set
    v[4] = math.nan
    l = Rows(6, experts, TYPES[dtype][0], fill=v)
    ids, weights, dl, _ = check(l, 6, experts, 3, ALL, dtype, 1.0, True)
    assert ids[1, :2].tolist() == [13, 4] and ids[2, 0] == 9 and ids[3, 0] == 2 and ids[4].tolist() == [0, 1, 2]
    clean = torch.tensor([0, 5], device="cuda")
    assert torch.isnan(weights[1:5]).any(1).all() and torch.isfinite(weights[clean]).all()
    assert torch.isnan(dl[1:5]).any(1).all() and torch.isfinite(dl[clean]).all()


@pytest.mark.parametrize("over", [ALL, CHOSEN])
@pytest.mark.parametrize("experts", [16, 90, 1100])
def test_gradient_of_given_ids(cuda_ok, experts, over):
    """Ids out of range add nothing, an expert named twice takes both gradients,
    whatever the order."""
    rows, k, gen = 40, 6, gen_of(6)
    l = Rows(rows, experts, torch.float32, fill=torch.randn(rows, experts, generator=gen, device="cuda"))
    ids = torch.randint(-2, min(experts + 3, 12), (rows, k), generator=gen, device="cuda").int()
    ids[0], ids[1] = 3, torch.tensor([experts, -1, 1 << 30, -(1 << 30), 5, 5])
    _, _, dl, dw = check(l, rows, experts, k, over, "f32", -0.75, True, ids=ids)
    against_fp64(l.t, k, over, "f32", -0.75, None, None, dl, dw, forward_ids=ids)


def test_differences(cuda_ok):
    """The gradient against central differences of the fp64 weights: with a step
    of 1e-4 their error is about 1e-8 and 1e-12 / 1e-4 of the terms."""
    rows, experts, k, gen = 7, 24, 4, gen_of(7)
    v = torch.randn(rows, experts, generator=gen, device="cuda")
    for over in (ALL, CHOSEN):
        l = Rows(rows, experts, torch.float32, fill=v)
        ids, _, dl, dw = check(l, rows, experts, k, over, "f32", 2.0, True)
        ids = ids.long()
        loss = lambda x: (2.0 * at(softmax(x, ids, over), ids) * dw.double()).sum(1)  # noqa: E731
        for e in range(experts):
            step = torch.zeros(experts, dtype=torch.float64, device="cuda")
            step[e] = 1e-4
            slope = (loss(v.double() + step) - loss(v.double() - step)) / 2e-4
            within(dl[:, e], slope, 2e-6 * (1 + dw.abs().sum(1).double()), f"expert {e}")


@pytest.mark.parametrize("experts", [64, 1100])
def test_gradient_in_place(cuda_ok, experts):
    rows, k = 50, 4
    v = torch.randn(rows, experts, generator=gen_of(8), device="cuda")
    l = Rows(rows, experts, torch.float32, fill=v)
    ids, _, dl, dw = check(l, rows, experts, k, ALL, "f32", 1.0, True)
    d = G.router_desc(rows, experts, k)
    G.goldy_router_backward(d, l.ptr, ids.data_ptr(), dw.data_ptr(), l.ptr)
    torch.cuda.synchronize()
    assert torch.equal(l.t, dl)
