"""Bias gradient of experts that cover only part of the rows, above all of a
single one, with a workspace that earlier calls have used: behind its counters it
holds NaN here, so that a partial sum that this call has not written shows.

A term passes at most (rows of its group) + 20 rounded additions (a lane's rows,
lanes, warps, slices, the sum that it is added to); an activation's slope is at
most 1.13 and good to 1e-6 (1 + |z|).
"""
import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from test_gpu_linear import ACTS, NAN, check, gen_of, matrix, offsets_of, ptr, slope64, spans, workspace

pytestmark = pytest.mark.gpu

PARTLY = [(1000, [20], 300), (1000, [0], 0), (1000, [0], 7), (1000, [0], 1000), (5000, [4000], 1000), (3000, [1], 2999),
          (3000, [1], 0), (64, [64], 0), (64, [63], 1), (4097, [2048], 1024), (300, [0, 20, 0], 100),
          (5000, [1, 0, 2000, 3], 900), (3000, [2] * 200, 17)]


@pytest.mark.parametrize("rows,counts,first", PARTLY)
@pytest.mark.parametrize("n", [8, 200, 1024])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_experts_with_part_of_the_rows(cuda_ok, rows, counts, first, n, act):
    gen, groups = gen_of(rows + first), len(counts)
    dy = matrix(gen, rows, n)
    z = matrix(gen, rows, n) if act != "none" else None
    dz = torch.full_like(dy, NAN) if act != "none" else None
    live = torch.zeros(rows, dtype=torch.bool, device="cuda")
    live[first:first + sum(counts)] = True
    dy[~live] = float("inf")                       # rows of no expert
    d = G.linear_desc(rows, 64, n, groups=groups, act=ACTS[act])
    ws, off = workspace(d), offsets_of(counts, first)
    db = torch.full((groups, n), NAN, device="cuda")
    for accumulate in (False, True):
        before = db.double().clone()
        ws[65536:].view(torch.float32).fill_(NAN)
        G.goldy_linear_bias_grad(d, ptr(dy), ptr(db), z=ptr(z), dz=ptr(dz), accumulate=accumulate, offsets=ptr(off),
                                 workspace=ptr(ws), workspace_bytes=ws.numel(),
                                 stream=torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert not ws[:65536].any(), "counters are not zero after the call"
        for e, lo, hi in spans(rows, counts, first):
            g, err = dy[lo:hi].double(), torch.zeros(hi - lo, n, device="cuda", dtype=torch.float64)
            if act != "none":
                z64 = z[lo:hi].double()
                err = 1e-6 * (1 + z64.abs()) * g.abs()
                g = g * slope64(z64, act)
            ref = g.sum(0) + (before[e] if accumulate else 0)
            bound = (hi - lo + 20) * 2.0 ** -24 * (g.abs().sum(0) + (before[e].abs() if accumulate else 0)) + err.sum(0)
            check(db[e], ref, bound + 1e-30, f"db of expert {e}")
        if dz is not None:
            assert torch.isnan(dz[~live].float()).all(), "a row of no expert was written"
