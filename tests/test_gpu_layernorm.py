"""Layer norm on the GPU against its definition in fp64.

Bounds: u = 2^-24 is the fp32 unit roundoff; a bf16 result adds 2^-8 of itself.
A sum over n elements passes at most `depth` rounded additions on any path
(values of a thread, 5 lane exchanges, up to 16 warps).  The mean is then off
by at most (depth + 1) u mean|x|, a difference x - mean by that and one rounding
of x, and rstd by half the relative error of the sum of squares plus a few
units of the square root.
"""
import pytest
import torch

from paper_2409_02227_gb300 import goldy as G

pytestmark = pytest.mark.gpu

TORCH = {G.GOLDY_BF16: torch.bfloat16, G.GOLDY_F32: torch.float32}
BF16, F32 = G.GOLDY_BF16, G.GOLDY_F32
U = 2.0 ** -24
NAN = float("nan")


def depth_of(n):
    return (16 if n <= 4096 else 32 if n <= 16384 else -(-n // 512)) + 5 + 16


def padded(t, ld, dtype):
    b = torch.full((t.shape[0], ld), NAN, device="cuda", dtype=TORCH[dtype])
    b[:, :t.shape[1]] = t
    return b[:, :t.shape[1]]


def inputs(rows, n, dtype, param, ld, seed, affine=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = padded(rnd(rows, n) * 2 + rnd(rows, 1) * 3 + 0.5, ld, dtype)
    dy = padded(rnd(rows, n), ld, dtype)
    gamma = (1 + 0.3 * rnd(n)).to(TORCH[param]) if affine else None
    beta = rnd(n).to(TORCH[param]) if affine else None
    return x, dy, gamma, beta


def ptr(t):
    return 0 if t is None else t.data_ptr()


def stream():
    return torch.cuda.current_stream().cuda_stream


def check(got, ref, tol, what):
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got.double() - ref).abs() - tol
    assert not (over > 0).any(), f"{what}: {float(over.max()):.3e} over its bound, {int((over > 0).sum())} elements"


def rounding(ref, dtype):
    return ref.abs() * (2.0 ** -8 if dtype == BF16 else 2.0 ** -22) + 1e-37


def forward(x, gamma, beta, dtype, param, eps=1e-5, stats=True, in_place=False):
    rows, n = x.shape
    y = x if in_place else torch.full((rows + 2, x.stride(0)), NAN, device="cuda", dtype=TORCH[dtype])[:, :n]
    mean = torch.full((rows,), NAN, device="cuda") if stats else None
    rstd = torch.full((rows,), NAN, device="cuda") if stats else None
    d = G.layernorm_desc(rows, n, dtype=dtype, param_dtype=param, eps=eps, ldx=x.stride(0), ldy=y.stride(0))
    G.goldy_layernorm_forward(d, ptr(x), ptr(gamma), ptr(beta), ptr(y), ptr(mean), ptr(rstd), stream())
    torch.cuda.synchronize()
    return y, mean, rstd


def check_forward(x64, y, mean, rstd, gamma, beta, dtype, eps=1e-5):
    rows, n = x64.shape
    m = x64.mean(1, keepdim=True)
    var = ((x64 - m) ** 2).mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    depth = depth_of(n)
    e = (depth + 1) * U * x64.abs().mean(1, keepdim=True) + 2 * U * x64.abs().max(1, keepdim=True).values
    rel = (depth + 4) * U + 2 * e * r + 2.0 ** -21
    xhat = (x64 - m) * r
    ga = gamma.double().abs() if gamma is not None else 1.0
    ref = xhat * (gamma.double() if gamma is not None else 1.0) + (beta.double() if beta is not None else 0.0)
    tol = ga * (e * r + xhat.abs() * rel) + 4 * U * (ref.abs() + ga * xhat.abs() + (beta.double().abs() if beta is not None else 0))
    check(y[:rows], ref, 1.01 * tol + 1.01 * rounding(ref, dtype), "Y")
    if mean is not None:
        check(mean, m[:, 0], e[:, 0] + 1e-37, "mean")
        check(rstd, r[:, 0], r[:, 0] * rel[:, 0], "rstd")


SIZES = [(1, 1), (3, 2), (2, 7), (5, 16), (150, 31), (33, 33), (1, 500), (1000, 512), (4, 513), (77, 1000), (300, 1023),
         (2000, 1024), (9, 1025), (129, 2048), (310, 2500), (1, 4096), (700, 4096), (20, 5000), (40, 8192), (3, 8193),
         (160, 10001), (30, 16384), (5, 16390)]


@pytest.mark.parametrize("rows,n", SIZES)
@pytest.mark.parametrize("dtype,param", [(BF16, BF16), (F32, F32), (BF16, F32)])
def test_forward(cuda_ok, rows, n, dtype, param):
    x, _, gamma, beta = inputs(rows, n, dtype, param, n, rows + n)
    y, mean, rstd = forward(x, gamma, beta, dtype, param)
    check_forward(x.double(), y, mean, rstd, gamma, beta, dtype)
    whole = y._base
    assert torch.isnan(whole[rows:]).all()


@pytest.mark.parametrize("rows,n,ld", [(20, 100, 104), (20, 96, 97), (7, 1000, 1003), (50, 2048, 2056), (6, 8193, 8200)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_forward_strides(cuda_ok, rows, n, ld, dtype):
    x, _, gamma, beta = inputs(rows, n, dtype, F32, ld, 1)
    y, mean, rstd = forward(x, gamma, beta, dtype, F32)
    check_forward(x.double(), y, mean, rstd, gamma, beta, dtype)
    assert torch.isnan(y._base[:, n:]).all(), "padding was written"
    x64 = x.double()
    y, mean, rstd = forward(x, None, None, dtype, F32, in_place=True, stats=False)
    check_forward(x64, y, None, None, None, None, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [64, 1000, 4096, 9000])
def test_forward_hard_rows(cuda_ok, dtype, n):
    """A constant row, a row far from zero, a tiny row, one outlier."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    x = torch.randn(5, n, generator=g, device="cuda")
    x[0] = 3.0
    x[1] = x[1] * 0.5 + 1000
    x[2] *= 1e-4
    x[3, n // 2] = 3e4
    x = x.to(TORCH[dtype])
    y, mean, rstd = forward(x, None, None, dtype, F32)
    check_forward(x.double(), y, mean, rstd, None, None, dtype)


def test_forward_nan_stays_in_its_row(cuda_ok):
    x, _, gamma, beta = inputs(40, 1000, BF16, BF16, 1000, 4)
    clean, _, _ = forward(x, gamma, beta, BF16, BF16)
    x[7, 3], x[21, 999] = NAN, float("inf")
    dirty, _, _ = forward(x, gamma, beta, BF16, BF16)
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[[7, 21]] = False
    assert torch.equal(clean[:40][keep], dirty[:40][keep])
    assert not torch.isfinite(dirty[[7, 21]].float()).any()


def backward(x, dy, gamma, mean, rstd, dtype, param, accumulate=False, start=None, want=(True, True)):
    rows, n = x.shape
    dx = torch.full((rows + 2, x.stride(0)), NAN, device="cuda", dtype=TORCH[dtype])[:, :n]
    dg, db = (torch.full((n,), NAN, device="cuda") if start is None else start.clone() for _ in range(2))
    d = G.layernorm_desc(rows, n, dtype=dtype, param_dtype=param, ldx=x.stride(0), ldy=dy.stride(0))
    ws = torch.zeros(max(G.goldy_layernorm_query(d), 256), dtype=torch.uint8, device="cuda")
    G.goldy_layernorm_backward(d, ptr(dy), ptr(x), ptr(gamma), ptr(mean), ptr(rstd), ptr(dx), ptr(dg) if want[0] else 0,
                               ptr(db) if want[1] else 0, ptr(ws), ws.numel(), stream(), accumulate=accumulate)
    torch.cuda.synchronize()
    assert not ws[:65536].any()
    return dx, dg, db


def check_backward(x, dy, gamma, mean, rstd, dx, dg, db, dtype, start=None):
    rows, n = x.shape
    depth = depth_of(n)
    x64, dy64, m, r = x.double(), dy.double(), mean.double()[:, None], rstd.double()[:, None]
    xhat = (x64 - m) * r
    exh = 3 * U * (x64.abs() + m.abs()) * r
    g = dy64 * (gamma.double() if gamma is not None else 1.0)
    s1, s2 = g.mean(1, keepdim=True), (g * xhat).mean(1, keepdim=True)
    ref = r * (g - s1 - xhat * s2)
    es1 = (depth + 4) * U * g.abs().mean(1, keepdim=True)
    es2 = (depth + 4) * U * (g * xhat).abs().mean(1, keepdim=True) + (g.abs() * exh).mean(1, keepdim=True)
    tol = r * (es1 + xhat.abs() * es2 + exh * s2.abs() + 4 * U * (g.abs() + s1.abs() + (xhat * s2).abs()))
    check(dx[:rows], ref, 1.01 * tol + 1.01 * rounding(ref, dtype), "dX")
    adds = -(-rows // 152) + 16 + 19 + 8
    for got, t, extra, what in ((dg, dy64 * xhat, (dy64.abs() * exh).sum(0), "dgamma"), (db, dy64, 0.0, "dbeta")):
        if got is None:
            continue
        first = start.double() if start is not None else 0.0
        bound = (adds + 2) * U * (t.abs().sum(0) + (start.double().abs() if start is not None else 0.0)) + extra + 1e-37
        check(got, t.sum(0) + first, bound, what)


@pytest.mark.parametrize("rows,n", SIZES)
@pytest.mark.parametrize("dtype,param", [(BF16, BF16), (F32, F32), (BF16, F32)])
def test_backward(cuda_ok, rows, n, dtype, param):
    x, dy, gamma, _ = inputs(rows, n, dtype, param, n, rows * n)
    mean = x.double().mean(1).float()
    rstd = (1 / torch.sqrt(x.double().var(1, unbiased=False) + 1e-5)).float()
    dx, dg, db = backward(x, dy, gamma, mean, rstd, dtype, param)
    check_backward(x, dy, gamma, mean, rstd, dx, dg, db, dtype)
    assert torch.isnan(dx._base[rows:]).all()
    start = torch.linspace(-1, 1, n, device="cuda")
    dx, dg, db = backward(x, dy, gamma, mean, rstd, dtype, param, accumulate=True, start=start)
    check_backward(x, dy, gamma, mean, rstd, dx, dg, db, dtype, start)


@pytest.mark.parametrize("rows,n,ld", [(20, 100, 104), (7, 1000, 1003), (50, 2048, 2056), (6, 8193, 8200)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_backward_strides_and_options(cuda_ok, rows, n, ld, dtype):
    x, dy, _, _ = inputs(rows, n, dtype, F32, ld, 1)
    mean, rstd = x.double().mean(1).float(), (1 / torch.sqrt(x.double().var(1, unbiased=False) + 1e-5)).float()
    for want in ((True, True), (True, False), (False, True), (False, False)):
        dx, dg, db = backward(x, dy, None, mean, rstd, dtype, F32, want=want)
        check_backward(x, dy, None, mean, rstd, dx, dg if want[0] else None, db if want[1] else None, dtype)
        assert torch.isnan(dx._base[:, n:]).all()
        assert want[0] or torch.isnan(dg).all()
        assert want[1] or torch.isnan(db).all()


def test_no_rows(cuda_ok):
    x, dy, gamma, _ = inputs(0, 100, BF16, BF16, 100, 1)
    mean = torch.empty(0, device="cuda")
    dx, dg, db = backward(x, dy, gamma, mean, mean, BF16, BF16)
    assert (dg == 0).all() and (db == 0).all()
    forward(x, gamma, gamma, BF16, BF16)


def test_gradient_against_differences(cuda_ok):
    """Directional central differences of the fp64 forward pass (error of the
    difference: h^2; of the fp32 gradient: 1e-5)."""
    rows, n, eps = 30, 257, 1e-5
    x, dy, gamma, beta = inputs(rows, n, F32, F32, n, 3)
    y, mean, rstd = forward(x, gamma, beta, F32, F32)
    dx, dg, db = backward(x, dy, gamma, mean, rstd, F32, F32)

    def loss(x, gamma, beta):
        m = x.mean(1, keepdim=True)
        return float((((x - m) / torch.sqrt(((x - m) ** 2).mean(1, keepdim=True) + eps) * gamma + beta) * dy.double()).sum())

    at, h = [t.double() for t in (x, gamma, beta)], 1e-4
    for i, grad in enumerate((dx[:rows], dg, db)):
        v = grad.double() / grad.double().norm()
        lo, hi = list(at), list(at)
        lo[i], hi[i] = at[i] - h * v, at[i] + h * v
        slope = (loss(*hi) - loss(*lo)) / (2 * h)
        assert abs(slope - float((grad.double() * v).sum())) < 1e-4 * abs(slope)


def test_same_bits_every_run(cuda_ok):
    x, dy, gamma, beta = inputs(3000, 1023, F32, F32, 1023, 3)
    y, mean, rstd = forward(x, gamma, beta, F32, F32)
    first = backward(x, dy, gamma, mean, rstd, F32, F32)
    again = backward(x, dy, gamma, mean, rstd, F32, F32)
    for a, b in zip(first, again):
        assert torch.equal(a[:3000] if a.dim() == 2 else a, b[:3000] if b.dim() == 2 else b)


def test_long_strides(cuda_ok):
    """Element offsets past 2^31."""
    rows, n, ld = 4, 300, 1 << 30
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.empty(rows * ld, device="cuda", dtype=torch.bfloat16).view(rows, ld)[:, :n]
    x.copy_(torch.randn(rows, n, generator=g, device="cuda"))
    y = torch.empty(rows, n, device="cuda", dtype=torch.bfloat16)
    d = G.layernorm_desc(rows, n, param_dtype=F32, ldx=ld)
    G.goldy_layernorm_forward(d, ptr(x), 0, 0, ptr(y), 0, 0, stream())
    torch.cuda.synchronize()
    check_forward(x.double(), y, None, None, None, None, BF16)
