"""Results that the linear layer's calls may write over one of their inputs: the
same bits as in a matrix of its own."""
import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from test_gpu_linear import ACTS, BF16, F32, NAN, TORCH, finish, gen_of, matrix, offsets_of, ptr, workspace

pytestmark = pytest.mark.gpu

# one CTA's tiles, splits of the reduction, pairs, groups; rows of any alignment
SIZES = [(1, 1024, 512, 0, None), (37, 4096, 1024, 0, None), (300, 640, 700, 1, None), (513, 96, 131, 0, None),
         (2048, 512, 1024, 0, None), (1000, 256, 520, 3, [0, 513, 87, 0, 400])]


def residual(gen, rows, n, pad, dtype):
    t = torch.full((rows, n + pad), NAN, device="cuda", dtype=TORCH[dtype])
    t[:, :n] = torch.randn(rows, n, generator=gen, device="cuda")
    return t[:, :n]


@pytest.mark.parametrize("rows,k,n,pad,counts", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_forward_onto_its_residual(cuda_ok, rows, k, n, pad, counts, dtype, act):
    gen, groups = gen_of(rows), len(counts or [])
    x, w = matrix(gen, rows, k), matrix(gen, k, n, None, k ** -0.5, (groups,) if groups else ())
    r = residual(gen, rows, n, pad, dtype)
    d = G.linear_desc(rows, k, n, groups=groups, act=ACTS[act], y_dtype=dtype, ldx=x.stride(0), ldw=w.stride(-2),
                      ldy=r.stride(0), ldr=r.stride(0))
    ws, off = workspace(d), offsets_of(counts)
    kw = dict(offsets=ptr(off), workspace=ptr(ws), workspace_bytes=ws.numel(), stream=torch.cuda.current_stream().cuda_stream)
    y = torch.full((rows, n + pad), NAN, device="cuda", dtype=TORCH[dtype])[:, :n]
    G.goldy_linear_forward(d, ptr(x), ptr(w), ptr(y), residual=ptr(r), **kw)
    G.goldy_linear_forward(d, ptr(x), ptr(w), ptr(r), residual=ptr(r), **kw)
    finish(ws)
    assert torch.isfinite(y.float()).all() and torch.equal(y, r)


@pytest.mark.parametrize("rows,n,k,pad,counts", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_input_gradient_onto_its_residual(cuda_ok, rows, n, k, pad, counts, dtype, act):
    gen, groups = gen_of(rows), len(counts or [])
    dy, w = matrix(gen, rows, n), matrix(gen, k, n, None, n ** -0.5, (groups,) if groups else ())
    z = matrix(gen, rows, k, k + pad) if act != "none" else None
    r = residual(gen, rows, k, pad, dtype)
    d = G.linear_desc(rows, k, n, groups=groups, act_x=ACTS[act], dx_dtype=dtype, lddx=r.stride(0), ldr=r.stride(0),
                      ldw=w.stride(-2), ldy=dy.stride(0), ldz=z.stride(0) if z is not None else 0)
    ws, off = workspace(d), offsets_of(counts)
    kw = dict(offsets=ptr(off), workspace=ptr(ws), workspace_bytes=ws.numel(), stream=torch.cuda.current_stream().cuda_stream)
    dx = torch.full((rows, k + pad), NAN, device="cuda", dtype=TORCH[dtype])[:, :k]
    G.goldy_linear_input_grad(d, ptr(dy), ptr(w), ptr(dx), z=ptr(z), residual=ptr(r), **kw)
    G.goldy_linear_input_grad(d, ptr(dy), ptr(w), ptr(r), z=ptr(z), residual=ptr(r), **kw)
    finish(ws)
    assert torch.isfinite(dx.float()).all() and torch.equal(dx, r)
