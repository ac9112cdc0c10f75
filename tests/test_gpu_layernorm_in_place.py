"""Layer norm written over its input, and its gradient over either of its inputs:
the same bits as in a matrix of its own, by every kernel (teams of all sizes, rows
off 16 bytes, clusters, streamed rows)."""
import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from test_gpu_layernorm import BF16, F32, NAN, TORCH, ptr, stream

pytestmark = pytest.mark.gpu

SIZES = [(700, 30, 0), (300, 257, 0), (500, 1000, 3), (2000, 1023, 0), (400, 4096, 0), (300, 8192, 0), (50, 9000, 8),
         (20, 12289, 0), (3, 60000, 0), (160, 70000, 0), (2, 140001, 0)]


@pytest.mark.parametrize("rows,n,pad", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_over_an_input(cuda_ok, rows, n, pad, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    fresh = lambda: torch.full((rows, n + pad), NAN, device="cuda", dtype=TORCH[dtype])[:, :n]  # noqa: E731
    x, dy = fresh(), fresh()
    x.copy_(rnd(rows, n) + 0.5)
    dy.copy_(rnd(rows, n))
    copy = lambda t: fresh().copy_(t)  # noqa: E731
    gamma, beta = 1 + 0.3 * rnd(n), rnd(n)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    d = G.layernorm_desc(rows, n, dtype=dtype, param_dtype=F32, ldx=n + pad, ldy=n + pad)

    y, place = fresh(), copy(x)
    G.goldy_layernorm_forward(d, ptr(x), ptr(gamma), ptr(beta), ptr(y), ptr(mean), ptr(rstd), stream())
    G.goldy_layernorm_forward(d, ptr(place), ptr(gamma), ptr(beta), ptr(place), 0, 0, stream())
    torch.cuda.synchronize()
    assert torch.isfinite(y.float()).all() and torch.equal(y, place)

    ws = torch.zeros(G.goldy_layernorm_query(d), dtype=torch.uint8, device="cuda")
    results = []
    for which in ("own", "dy", "x"):
        a, b, dx = copy(dy), copy(x), fresh()
        dx = {"own": dx, "dy": a, "x": b}[which]
        dg, db = torch.full((n,), NAN, device="cuda"), torch.full((n,), NAN, device="cuda")
        G.goldy_layernorm_backward(d, ptr(a), ptr(b), ptr(gamma), ptr(mean), ptr(rstd), ptr(dx), ptr(dg), ptr(db), ptr(ws),
                                   ws.numel(), stream())
        torch.cuda.synchronize()
        results.append((dx, dg, db))
    for other in results[1:]:
        for p, q in zip(results[0], other):
            assert torch.isfinite(p.float()).all() and torch.equal(p, q)
