"""Layer norm of rows that start on any element's boundary, against its
definition in fp64 (bounds: test_gpu_layernorm.py)."""
import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from test_gpu_layernorm import BF16, F32, NAN, TORCH, check_backward, check_forward, ptr, stream

pytestmark = pytest.mark.gpu


def view(buf, first, rows, n, ld):
    return torch.as_strided(buf, (rows, n), (ld, 1), first)


@pytest.mark.parametrize("rows,n", [(1, 1), (9, 2), (7, 3), (50, 31), (5, 32), (33, 33), (6, 62), (6, 64), (77, 65), (40, 255),
                                    (37, 513), (310, 1000), (9, 1023), (9, 2049), (20, 4095), (11, 8191), (3, 8193),
                                    (2, 16383), (3, 20001)])
@pytest.mark.parametrize("first,pad", [((0, 1, 1), (0, 0)), ((1, 0, 1), (1, 0)), ((3, 5, 0), (0, 3)), ((1, 1, 1), (2, 2))])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_any_start(cuda_ok, rows, n, first, pad, dtype):
    ldx, ldy = n + pad[0], n + pad[1]
    g = torch.Generator(device="cuda")
    g.manual_seed(n + sum(first))
    fresh = lambda ld: torch.full((rows * ld + 16,), NAN, device="cuda", dtype=TORCH[dtype])  # noqa: E731
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, dy = view(fresh(ldx), first[0], rows, n, ldx), view(fresh(ldy), first[1], rows, n, ldy)
    x.copy_(rnd(rows, n) + 0.5)
    dy.copy_(rnd(rows, n))
    gamma, beta = 1 + 0.3 * rnd(n), rnd(n)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    d = G.layernorm_desc(rows, n, dtype=dtype, param_dtype=F32, ldx=ldx, ldy=ldy)

    whole = fresh(ldy)
    y = view(whole, first[2], rows, n, ldy)
    G.goldy_layernorm_forward(d, ptr(x), ptr(gamma), ptr(beta), ptr(y), ptr(mean), ptr(rstd), stream())
    torch.cuda.synchronize()
    check_forward(x.double(), y, mean, rstd, gamma, beta, dtype)
    y.fill_(NAN)
    assert torch.isnan(whole).all(), "written outside the rows"

    whole = fresh(ldx)
    dx = view(whole, first[2], rows, n, ldx)
    dg, db = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ws = torch.zeros(G.goldy_layernorm_query(d), dtype=torch.uint8, device="cuda")
    G.goldy_layernorm_backward(d, ptr(dy), ptr(x), ptr(gamma), ptr(mean), ptr(rstd), ptr(dx), ptr(dg), ptr(db), ptr(ws),
                               ws.numel(), stream())
    torch.cuda.synchronize()
    check_backward(x, dy, gamma, mean, rstd, dx, dg, db, dtype)
    dx.fill_(NAN)
    assert torch.isnan(whole).all(), "written outside the rows"

    x64 = x.double()
    d = G.layernorm_desc(rows, n, dtype=dtype, param_dtype=F32, ldx=ldx, ldy=ldx)
    G.goldy_layernorm_forward(d, ptr(x), ptr(gamma), ptr(beta), ptr(x), 0, 0, stream())
    torch.cuda.synchronize()
    check_forward(x64, x, None, None, gamma, beta, dtype)
