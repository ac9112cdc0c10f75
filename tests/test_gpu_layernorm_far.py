"""Layer norm backwards for rows far from zero, against its definition in fp64
for the given mean and rstd.

Bounds: u = 2^-24.  Subtracting first, x - mean is off by u of itself, and
xhat = (x - mean) rstd by 2 u of itself, however large mean is; 3 u here.  A sum
over a row passes at most `depth` rounded additions, a sum over rows at most one
per row and 45 (threads, teams, CTAs), as in test_gpu_layernorm.py.
"""
import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from test_gpu_layernorm import BF16, F32, TORCH, U, backward, check, depth_of, rounding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [30, 257, 1000, 4096, 8192, 9000, 60001, 70000])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_far_from_zero(cuda_ok, n, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    far = torch.tensor([0.0, 10.0, -100.0, 2000.0, -3.0, 500.0], device="cuda")[:, None]   # in deviations
    rows = far.shape[0]
    x = (0.5 * (rnd(rows, n) + far)).to(TORCH[dtype])
    dy, gamma = rnd(rows, n).to(TORCH[dtype]), 1 + 0.3 * rnd(n)
    mean = x.double().mean(1).float()
    rstd = (1 / torch.sqrt(x.double().var(1, unbiased=False) + 1e-5)).float()
    dx, dg, db = backward(x, dy, gamma, mean, rstd, dtype, F32)

    depth = depth_of(n)
    m, r = mean.double()[:, None], rstd.double()[:, None]
    xhat = (x.double() - m) * r
    exh = 3 * U * xhat.abs()
    g = dy.double() * gamma.double()
    s1, s2 = g.mean(1, keepdim=True), (g * xhat).mean(1, keepdim=True)
    ref = r * (g - s1 - xhat * s2)
    es1 = (depth + 4) * U * g.abs().mean(1, keepdim=True)
    es2 = (depth + 4) * U * (g * xhat).abs().mean(1, keepdim=True) + (g.abs() * exh).mean(1, keepdim=True)
    tol = r * (es1 + xhat.abs() * es2 + exh * s2.abs() + 4 * U * (g.abs() + s1.abs() + (xhat * s2).abs()))
    check(dx[:rows], ref, 1.01 * tol + 1.01 * rounding(ref, dtype), "dX")
    t = dy.double() * xhat
    check(dg, t.sum(0), (rows + 45) * U * t.abs().sum(0) + (dy.double().abs() * exh).sum(0) + 1e-37, "dgamma")
    check(db, dy.double().sum(0), (rows + 45) * U * dy.double().abs().sum(0) + 1e-37, "dbeta")
