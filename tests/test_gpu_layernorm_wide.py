"""Layer norm of rows that clusters of CTAs share, against its definition in
fp64 (bounds: test_gpu_layernorm.py).

A path of additions passes 16 or 32 values of a thread, 5 + 4 exchanges and 8
CTAs, below depth_of(n).  For dgamma and dbeta it passes at most every row of a
cluster (the 160 rows here are shared by many, the others have at most 50), then
the partial rows: below check_backward's count.
"""
import pytest
import torch

import test_gpu_layernorm as base
from paper_2409_02227_gb300 import goldy as G
from test_gpu_layernorm import BF16, F32, backward, check_backward, check_forward, forward, inputs

pytestmark = pytest.mark.gpu

# at and around the limits of 2, 4 and 8 CTAs, backwards and forwards, and beyond them
WIDE = [(3, 8200), (160, 12288), (5, 12289), (2, 16376), (4, 16385), (1, 32768), (3, 32770), (2, 65536), (2, 65537),
        (1, 131072), (2, 131073)]


@pytest.mark.parametrize("rows,n", WIDE)
@pytest.mark.parametrize("dtype,param", [(BF16, BF16), (F32, F32), (BF16, F32)])
def test_wide_rows(cuda_ok, rows, n, dtype, param):
    x, dy, gamma, beta = inputs(rows, n, dtype, param, n + 8, n)
    y, mean, rstd = forward(x, gamma, beta, dtype, param)
    check_forward(x.double(), y, mean, rstd, gamma, beta, dtype)
    assert torch.isnan(y._base[rows:]).all() and torch.isnan(y._base[:, n:]).all()
    start = torch.linspace(-1, 1, n, device="cuda")
    for begin in (None, start):
        dx, dg, db = backward(x, dy, gamma, mean, rstd, dtype, param, accumulate=begin is not None, start=begin)
        check_backward(x, dy, gamma, mean, rstd, dx, dg, db, dtype, begin)
        assert torch.isnan(dx._base[rows:]).all() and torch.isnan(dx._base[:, n:]).all()


def test_wide_rows_in_an_sm_partition(cuda_ok, monkeypatch):
    part = G.goldy_partition_create(16, 1)
    _, streams = G.goldy_partition_query(part, 1)
    # (behind everything asked of the current stream)
    monkeypatch.setattr(base, "stream", lambda: (torch.cuda.synchronize(), streams[0])[1])
    for rows, n in ((50, 12288), (9, 60000)):
        x, dy, gamma, beta = inputs(rows, n, BF16, F32, n, rows)
        y, mean, rstd = forward(x, gamma, beta, BF16, F32)
        check_forward(x.double(), y, mean, rstd, gamma, beta, BF16)
        dx, dg, db = backward(x, dy, gamma, mean, rstd, BF16, F32)
        check_backward(x, dy, gamma, mean, rstd, dx, dg, db, BF16)
    part.close()
