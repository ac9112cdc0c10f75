"""Bias gradient through every activation, its dZ in a matrix of its own and in
dY's place (bounds: test_gpu_linear.py)."""
import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from test_gpu_linear import (ACTS, BF16, NAN, check, finish, gen_of, matrix, offsets_of, ptr, round_tol, slope64, spans,
                             workspace)

pytestmark = pytest.mark.gpu

REAL = [a for a in ACTS if a != "none"]


def run(dy, z, dz, n, act, counts=None, first=0):
    d = G.linear_desc(dy.shape[0], 64, n, groups=len(counts or []), act=ACTS[act], ldy=dy.stride(0), ldz=z.stride(0))
    ws, off = workspace(d), offsets_of(counts, first)
    db = torch.full((max(1, len(counts or [])), n), NAN, device="cuda")
    G.goldy_linear_bias_grad(d, ptr(dy), ptr(db), z=ptr(z), dz=ptr(dz), offsets=ptr(off), workspace=ptr(ws),
                             workspace_bytes=ws.numel(), stream=torch.cuda.current_stream().cuda_stream)
    finish(ws)
    return db


# widths with and without whole 16-byte pieces, rows of several passes and slices
@pytest.mark.parametrize("rows,n,ld,counts,first", [(1, 8, 8, None, 0), (70, 257, 264, None, 0), (33, 77, 77, None, 0),
                                                    (1000, 1024, 1024, None, 0), (4097, 96, 104, None, 0),
                                                    (300, 200, 200, [17, 0, 128, 1, 33, 64], 20), (900, 65, 72, [500], 100)])
@pytest.mark.parametrize("act", REAL)
def test_activation(cuda_ok, rows, n, ld, counts, first, act):
    gen = gen_of(rows + n)
    dy, z = matrix(gen, rows, n, ld), matrix(gen, rows, n, ld, 2.0)
    z[0, :3] = torch.tensor([0.0, -0.0, 1.0]).bfloat16()
    dz = torch.full_like(dy._base, NAN)[:, :n] if dy._base is not None else torch.full_like(dy, NAN)
    assert dz.stride(0) == dy.stride(0)
    db = run(dy, z, dz, n, act, counts, first)
    for e, lo, hi in spans(rows, counts, first):
        z64, g = z[lo:hi].double(), dy[lo:hi].double()
        err = 1e-6 * (1 + z64.abs()) * g.abs()
        g = g * slope64(z64, act)
        if hi > lo:
            check(dz[lo:hi], g, err + round_tol(g, BF16) * 1.01, f"dZ of group {e}")
        check(db[e], g.sum(0), (hi - lo + 20) * 2.0 ** -24 * g.abs().sum(0) + err.sum(0) + 1e-30, f"db of group {e}")
    place = dy.clone(memory_format=torch.preserve_format) if ld == n else torch.cat([dy, dy[:, :1].expand(rows, ld - n)], 1)[:, :n]
    again = run(place, z, place, n, act, counts, first)
    assert torch.equal(again, db)
    for e, lo, hi in spans(rows, counts, first):
        assert torch.equal(place[lo:hi], dz[lo:hi])
    gone = torch.ones(rows, dtype=torch.bool, device="cuda")
    for e, lo, hi in spans(rows, counts, first):
        gone[lo:hi] = False
    assert torch.equal(place[gone], dy[gone])


@pytest.mark.parametrize("act", REAL)
def test_saturated_slopes(cuda_ok, act):
    """Far from 0 a slope is 0 or 1, whatever z^3 and exp(z) come to: silu's at
    -60 the farthest from it, by 60 exp(-60) = 5.3e-25."""
    far = torch.tensor([60.0, 1e4, 1e19, 3e30, 3e38], device="cuda").bfloat16()
    z = torch.cat([far, -far]).repeat(3, 1)[:, :10].contiguous()
    dy = torch.full_like(z, 3.0)
    dz = torch.full_like(z, NAN)
    db = run(dy, z, dz, 10, act)
    want = torch.tensor([3.0] * 5 + [0.0] * 5, device="cuda").repeat(3, 1)
    assert ((dz.float() - want).abs() <= 3 * 5.3e-25).all()
    assert ((db[0] - want.sum(0)).abs() <= 9 * 5.3e-25).all()
