"""Linear-layer operators on the GPU against their definitions in fp64.

Bounds (none is fitted to a result).  A product's inputs are bf16, so its
exact terms are fp32 numbers; the tensor core adds 16 reduction elements per
step and truncates the fp32 accumulator, an error of at most 2^-22 of the sum
of absolute terms S per step.  With steps(K) steps in one accumulator (bf16
results: K / 16; fp32 results: 32 and one rounded addition per 512) the
accumulated value is off by at most (steps + 2) 2^-22 S.  An activation's slope
is at most 1.13 and its fp32 evaluation is good to 1e-6 (1 + |z|).  A bf16
result adds 2^-8 of itself (rounding to nearest with 8 significant bits), an fp32
result 2^-22.
"""
import math

import pytest
import torch

from paper_2409_02227_gb300 import goldy as G

pytestmark = pytest.mark.gpu

ACTS = {"none": G.GOLDY_ACT_NONE, "relu": G.GOLDY_ACT_RELU, "gelu": G.GOLDY_ACT_GELU,
        "gelu_tanh": G.GOLDY_ACT_GELU_TANH, "silu": G.GOLDY_ACT_SILU}
TORCH = {G.GOLDY_BF16: torch.bfloat16, G.GOLDY_F32: torch.float32}
BF16, F32 = G.GOLDY_BF16, G.GOLDY_F32
NAN = float("nan")


def act64(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def slope64(z, act):
    z = z.detach().clone().requires_grad_(True)
    act64(z, act).sum().backward()
    g = z.grad
    if act == "relu":
        g = torch.where(z > 0, 1.0, 0.0).double()
    return g.detach()


def matrix(gen, rows, cols, ld=None, scale=1.0, lead=(), fill=NAN):
    """bf16 matrix view whose padding holds NaN."""
    ld = (cols + 7) // 8 * 8 if ld is None else ld
    t = torch.full((*lead, rows, ld), fill, device="cuda", dtype=torch.bfloat16)
    t[..., :cols] = (torch.randn(*lead, rows, cols, generator=gen, device="cuda") * scale).bfloat16()
    return t[..., :cols]


def out_matrix(rows, cols, dtype, ld=None, lead=(), guard=0):
    """Result buffer: NaN everywhere, so that an unwritten element shows."""
    ld = cols if ld is None else ld
    return torch.full((*lead, rows + guard, ld), NAN, device="cuda", dtype=TORCH[dtype])[..., :cols]


def gen_of(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def spans(rows, counts, first=0):
    if counts is None:
        return [(0, 0, rows)]
    out, r = [], first
    for e, c in enumerate(counts):
        out.append((e, r, r + c))
        r += c
    assert r <= rows
    return out


def offsets_of(counts, first=0):
    if counts is None:
        return None
    o = [first]
    for c in counts:
        o.append(o[-1] + c)
    return torch.tensor(o, dtype=torch.int32, device="cuda")


def steps(k, dtype):
    if dtype == BF16:
        return k / 16
    return min(k, 512) / 16 + math.ceil(k / 512)


def round_tol(ref, dtype):
    return ref.abs() * (2.0 ** -8 if dtype == BF16 else 2.0 ** -22) + (1e-38 if dtype == F32 else 1e-38)


def check(got, ref, tol, what):
    assert torch.isfinite(got).all(), f"{what}: not finite ({int((~torch.isfinite(got)).sum())} elements)"
    over = (got.double() - ref).abs() - tol
    assert not (over > 0).any(), (f"{what}: off by {float((got.double() - ref).abs().max()):.3e}, "
                                  f"{float(over.max()):.3e} over its bound, {int((over > 0).sum())} elements")


def workspace(d):
    n = G.goldy_linear_query(d)
    return torch.zeros(max(n, 256), dtype=torch.uint8, device="cuda")


def finish(ws):
    torch.cuda.synchronize()
    assert G.goldy_device_error(clear=True) == 0
    assert not ws[:65536].any(), "counters are not zero after the call"


def ptr(t):
    return 0 if t is None else t.data_ptr()


def run_forward(rows, k, n, counts=None, first=0, act="none", bias=True, residual=False, save=False, y_dtype=BF16,
                bias_dtype=BF16, ldx=None, ldw=None, ldy=None, seed=0, poison=False):
    gen = gen_of(seed)
    groups = 0 if counts is None else len(counts)
    lead = (groups,) if groups else ()
    x = matrix(gen, rows, k, ldx)
    w = matrix(gen, k, n, ldw, max(k, 1) ** -0.5, lead)
    b = (0.5 * torch.randn(*lead, n, generator=gen, device="cuda")).to(TORCH[bias_dtype]) if bias else None
    r = torch.randn(rows, n, generator=gen, device="cuda").to(TORCH[y_dtype]) if residual else None
    covered = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for e, lo, hi in spans(rows, counts, first):
        covered[lo:hi] = True
    if poison:                       # rows of no group
        x[~covered] = NAN
    y = out_matrix(rows, n, y_dtype, ldy, guard=3)
    z = out_matrix(rows, n, BF16, None, guard=3) if save else None
    d = G.linear_desc(rows, k, n, groups=groups, act=ACTS[act], y_dtype=y_dtype, bias_dtype=bias_dtype,
                      ldx=x.stride(0), ldw=w.stride(-2), ldy=y.stride(0), ldz=n if save else 0, ldr=n if residual else 0)
    ws = workspace(d)
    off = offsets_of(counts, first)
    G.goldy_linear_forward(d, ptr(x), ptr(w), ptr(y), bias=ptr(b), residual=ptr(r), z=ptr(z), offsets=ptr(off),
                           workspace=ptr(ws), workspace_bytes=ws.numel(),
                           stream=torch.cuda.current_stream().cuda_stream)
    finish(ws)
    for e, lo, hi in spans(rows, counts, first):
        if lo == hi:
            continue
        xe, we = x[lo:hi].double(), (w[e] if groups else w).double()
        be = (b[e] if groups else b).double() if bias else torch.zeros(n, device="cuda", dtype=torch.float64)
        z64 = xe @ we + be
        s = xe.abs() @ we.abs() + be.abs()
        acc = (steps(k, y_dtype) + 2) * 2.0 ** -22 * s
        y64 = act64(z64, act) + (r[lo:hi].double() if residual else 0)
        tol = 1.2 * acc + (1e-6 * (1 + z64.abs()) if act != "none" else 0) + round_tol(y64, y_dtype) * 1.01 + 2.0 ** -22 * z64.abs()
        check(y[lo:hi], y64, tol, f"Y of group {e}")
        if save:
            check(z[lo:hi], z64, acc + round_tol(z64, BF16) * 1.01, f"Z of group {e}")
    gone = torch.ones(rows + 3, dtype=torch.bool, device="cuda")
    gone[:rows] = ~covered
    whole = y._base if y._base is not None else y
    assert torch.isnan(whole[gone]).all(), "a row of no group was written"
    if whole.shape[1] > n:
        assert torch.isnan(whole[:, n:]).all(), "padding of Y was written"
    return y


# rows around the tile and instruction granularities; features around 64 and 128
@pytest.mark.parametrize("rows,k,n", [(1, 64, 128), (1, 1024, 4096), (2, 8, 8), (15, 72, 136), (16, 64, 256), (17, 200, 129),
                                      (31, 1, 1), (33, 65, 40), (64, 512, 1024), (127, 130, 255), (129, 1000, 257),
                                      (255, 320, 640), (257, 96, 513), (511, 2048, 384), (700, 777, 1111),
                                      (2048, 256, 2048), (4097, 128, 264)])
@pytest.mark.parametrize("y_dtype", [BF16, F32])
def test_forward_sizes(cuda_ok, rows, k, n, y_dtype):
    run_forward(rows, k, n, y_dtype=y_dtype, seed=rows + k)


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("y_dtype", [BF16, F32])
@pytest.mark.parametrize("rows,k,n", [(5, 256, 320), (300, 640, 700)])
def test_forward_epilogue(cuda_ok, act, y_dtype, rows, k, n):
    run_forward(rows, k, n, act=act, residual=True, save=True, y_dtype=y_dtype, bias_dtype=F32, seed=3)
    run_forward(rows, k, n, act=act, bias=False, residual=False, save=True, y_dtype=y_dtype, seed=4)


def test_forward_strides(cuda_ok):
    run_forward(77, 100, 90, ldx=128, ldw=104, ldy=91, residual=True, save=True, act="gelu")
    run_forward(300, 1032, 520, ldx=1040, ldw=1000, ldy=1024, y_dtype=F32)
    run_forward(300, 1032, 520, ldx=1040, ldw=1000, ldy=523, y_dtype=F32, residual=True)


GROUPS = [
    (40, [40], 0), (64, [0, 30, 0, 34], 0), (64, [64, 0], 0), (100, [1, 1, 1, 0, 96], 1),
    (300, [17, 0, 128, 1, 33, 64], 20), (1000, [513, 487], 0), (1000, [0, 0, 256, 257, 255, 0, 100], 50),
    (500, [5] * 70, 3), (96, [0] * 40 + [50] + [0] * 31 + [40], 2), (30, [0, 0, 0], 7), (2000, [1500, 3, 2, 400], 0),
]


@pytest.mark.parametrize("rows,counts,first", GROUPS)
@pytest.mark.parametrize("y_dtype", [BF16, F32])
def test_forward_groups(cuda_ok, rows, counts, first, y_dtype):
    run_forward(rows, 136, 200, counts=counts, first=first, act="silu", y_dtype=y_dtype, save=True, poison=True)
    run_forward(rows, 512, 520, counts=counts, first=first, y_dtype=y_dtype, residual=True, poison=True)


def test_forward_groups_do_not_mix(cuda_ok):
    """A group whose rows hold infinities and NaN leaves the others alone."""
    rows, k, n, counts = 200, 128, 256, [50, 33, 60, 57]
    gen = gen_of(1)
    x, w = matrix(gen, rows, k), matrix(gen, k, n, None, k ** -0.5, (4,))
    off = offsets_of(counts)
    d = G.linear_desc(rows, k, n, groups=4)
    ws = workspace(d)
    y = out_matrix(rows, n, BF16)

    def go():
        G.goldy_linear_forward(d, ptr(x), ptr(w), ptr(y), offsets=ptr(off), workspace=ptr(ws), workspace_bytes=ws.numel(),
                               stream=torch.cuda.current_stream().cuda_stream)
        finish(ws)
        return y.clone()

    clean = go()
    x[50:83] = float("inf")
    x[60] = NAN
    dirty = go()
    assert torch.equal(clean[:50], dirty[:50]) and torch.equal(clean[83:], dirty[83:])
    assert not torch.isfinite(dirty[50:83].float()).all()


def run_input_grad(rows, k, n, counts=None, first=0, act="none", residual=False, dx_dtype=BF16, ldx=None, seed=0):
    gen = gen_of(seed)
    groups = 0 if counts is None else len(counts)
    lead = (groups,) if groups else ()
    dy = matrix(gen, rows, n)
    w = matrix(gen, k, n, None, max(n, 1) ** -0.5, lead)
    z = matrix(gen, rows, k, scale=1.5) if act != "none" else None
    r = torch.randn(rows, k, generator=gen, device="cuda").to(TORCH[dx_dtype]) if residual else None
    dx = out_matrix(rows, k, dx_dtype, ldx)
    d = G.linear_desc(rows, k, n, groups=groups, act_x=ACTS[act], dx_dtype=dx_dtype, lddx=dx.stride(0), ldw=w.stride(-2),
                      ldy=dy.stride(0), ldz=z.stride(0) if z is not None else 0, ldr=k if residual else 0)
    ws, off = workspace(d), offsets_of(counts, first)
    G.goldy_linear_input_grad(d, ptr(dy), ptr(w), ptr(dx), z=ptr(z), residual=ptr(r), offsets=ptr(off),
                              workspace=ptr(ws), workspace_bytes=ws.numel(),
                              stream=torch.cuda.current_stream().cuda_stream)
    finish(ws)
    for e, lo, hi in spans(rows, counts, first):
        if lo == hi:
            continue
        g, we = dy[lo:hi].double(), (w[e] if groups else w).double()
        p, s = g @ we.T, g.abs() @ we.abs().T
        acc = (steps(n, dx_dtype) + 2) * 2.0 ** -22 * s
        tol = acc
        if act != "none":
            z64 = z[lo:hi].double()
            sl = slope64(z64, act)
            tol = 1.2 * acc + 1e-6 * (1 + z64.abs()) * p.abs()
            p = p * sl
        if residual:
            p = p + r[lo:hi].double()
        check(dx[lo:hi], p, tol + round_tol(p, dx_dtype) * 1.01 + 2.0 ** -22 * s, f"dX of group {e}")
    return dx


@pytest.mark.parametrize("rows,k,n", [(1, 128, 64), (3, 129, 72), (17, 1000, 200), (130, 264, 520), (513, 700, 1030), (2048, 1024, 320)])
@pytest.mark.parametrize("dx_dtype", [BF16, F32])
@pytest.mark.parametrize("act,residual", [("none", False), ("gelu", True), ("silu", False), ("relu", True), ("gelu_tanh", False)])
def test_input_grad(cuda_ok, rows, k, n, dx_dtype, act, residual):
    run_input_grad(rows, k, n, act=act, residual=residual, dx_dtype=dx_dtype, seed=rows)


@pytest.mark.parametrize("rows,counts,first", GROUPS)
def test_input_grad_groups(cuda_ok, rows, counts, first):
    run_input_grad(rows, 200, 136, counts=counts, first=first, act="silu", ldx=203)
    run_input_grad(rows, 520, 512, counts=counts, first=first, dx_dtype=F32)


def run_weight_grad(rows, k, n, counts=None, first=0, dw_dtype=F32, accumulate=False, ldw=None, poison=True, seed=0):
    gen = gen_of(seed)
    groups = 0 if counts is None else len(counts)
    lead = (groups,) if groups else ()
    x, dy = matrix(gen, rows, k), matrix(gen, rows, n)
    if poison and groups:
        live = torch.zeros(rows, dtype=torch.bool, device="cuda")
        for e, lo, hi in spans(rows, counts, first):
            live[lo:hi] = True
        x[~live] = NAN
        dy[~live] = float("inf")
    ldw = n if ldw is None else ldw
    dw = out_matrix(k, n, dw_dtype, ldw, lead)
    if accumulate:
        dw[...] = torch.randn(*lead, k, n, generator=gen, device="cuda").to(TORCH[dw_dtype])
    before = dw.double().clone()
    stride_w = k * ldw
    d = G.linear_desc(rows, k, n, groups=groups, dw_dtype=dw_dtype, ldx=x.stride(0), ldw=ldw, ldy=dy.stride(0), stride_w=stride_w)
    ws, off = workspace(d), offsets_of(counts, first)
    G.goldy_linear_weight_grad(d, ptr(x), ptr(dy), ptr(dw), accumulate=accumulate, offsets=ptr(off), workspace=ptr(ws),
                               workspace_bytes=ws.numel(), stream=torch.cuda.current_stream().cuda_stream)
    finish(ws)
    for e, lo, hi in spans(rows, counts, first):
        xe, g = x[lo:hi].double(), dy[lo:hi].double()
        ref, s = xe.T @ g, xe.abs().T @ g.abs()
        got = dw[e] if groups else dw
        acc = (steps(hi - lo, dw_dtype) + 4) * 2.0 ** -22 * s
        if accumulate:
            ref = ref + (before[e] if groups else before)
        check(got, ref, acc + round_tol(ref, dw_dtype) * 1.01, f"dW of group {e}")
    return dw


@pytest.mark.parametrize("rows,k,n", [(1, 64, 64), (5, 130, 72), (63, 8, 136), (64, 256, 256), (65, 129, 257), (500, 333, 1000),
                                      (2000, 512, 264), (4096, 256, 512)])
@pytest.mark.parametrize("dw_dtype", [BF16, F32])
@pytest.mark.parametrize("accumulate", [False, True])
def test_weight_grad(cuda_ok, rows, k, n, dw_dtype, accumulate):
    run_weight_grad(rows, k, n, dw_dtype=dw_dtype, accumulate=accumulate, seed=rows)


@pytest.mark.parametrize("rows,counts,first", GROUPS)
@pytest.mark.parametrize("dw_dtype", [BF16, F32])
def test_weight_grad_groups(cuda_ok, rows, counts, first, dw_dtype):
    run_weight_grad(rows, 136, 200, counts=counts, first=first, dw_dtype=dw_dtype)
    run_weight_grad(rows, 264, 520, counts=counts, first=first, dw_dtype=dw_dtype, accumulate=True, ldw=528)


@pytest.mark.parametrize("size", [512, 1024])
def test_weight_grad_large_groups(cuda_ok, size):
    """Tiles of the CTA-pair kernel with every ragged tail length class."""
    counts = [1, 63, 64, 65, 190, 0, 7, 129, 300]
    run_weight_grad(sum(counts) + 9, size, 2 * size, counts=counts, first=4, dw_dtype=BF16)
    run_weight_grad(sum(counts) + 9, size, 2 * size, counts=counts, first=4, dw_dtype=F32)


@pytest.mark.parametrize("rows,k,n,counts", [(50, 75, 130, None), (1, 1001, 77, None), (700, 333, 515, None),
                                             (300, 131, 259, [100, 0, 37, 163])])
def test_rows_off_16_byte_boundaries(cuda_ok, rows, k, n, counts):
    """Packed rows of odd length, products in all directions."""
    gen = gen_of(k)
    groups = 0 if counts is None else len(counts)
    lead = (groups,) if groups else ()
    packed = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    x, w, dy = packed(rows, k), packed(*lead, k, n) * k ** -0.5, packed(rows, n)
    # base one element off as well
    x = torch.cat([x.new_full((1,), NAN), x.flatten()])[1:].view(rows, k)
    y, dx = out_matrix(rows, n, BF16), out_matrix(rows, k, BF16)
    dw = out_matrix(k, n, F32, lead=lead)
    d = G.linear_desc(rows, k, n, groups=groups, ldx=k, lddx=k, ldw=n, ldy=n, dw_dtype=F32)
    ws, off = workspace(d), offsets_of(counts)
    kw = dict(offsets=ptr(off), workspace=ptr(ws), workspace_bytes=ws.numel(), stream=torch.cuda.current_stream().cuda_stream)
    G.goldy_linear_forward(d, ptr(x), ptr(w), ptr(y), **kw)
    G.goldy_linear_input_grad(d, ptr(dy), ptr(w), ptr(dx), **kw)
    G.goldy_linear_weight_grad(d, ptr(x), ptr(dy), ptr(dw), **kw)
    finish(ws)
    for e, lo, hi in spans(rows, counts):
        xe, ge, we = x[lo:hi].double(), dy[lo:hi].double(), (w[e] if groups else w).double()
        for got, a, b, kk, dt in ((y[lo:hi], xe, we, k, BF16), (dx[lo:hi], ge, we.T, n, BF16),
                                  (dw[e] if groups else dw, xe.T, ge, hi - lo, F32)):
            ref = a @ b
            check(got, ref, (steps(kk, dt) + 4) * 2.0 ** -22 * (a.abs() @ b.abs()) + round_tol(ref, dt) * 1.01, f"group {e}")


@pytest.mark.parametrize("rows,n,counts,first", [(1, 8, None, 0), (70, 257, None, 0), (1000, 1024, None, 0), (4097, 96, None, 0)] +
                         [(r, 200, c, f) for r, c, f in GROUPS])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_bias_grad(cuda_ok, rows, n, counts, first, act):
    gen = gen_of(rows)
    groups = 0 if counts is None else len(counts)
    dy = matrix(gen, rows, n, n if act == "none" else None)
    z = matrix(gen, rows, n) if act != "none" else None
    dz = torch.full_like(dy, NAN) if act != "none" else None
    db = torch.full((max(1, groups), n), NAN, device="cuda")
    d = G.linear_desc(rows, 64, n, groups=groups, act=ACTS[act], ldw=(n + 7) // 8 * 8, ldy=dy.stride(0), ldz=z.stride(0) if z is not None else 0)
    if dz is not None:
        dz = torch.full((rows, dy.stride(0)), NAN, device="cuda", dtype=torch.bfloat16)[:, :n]
    ws, off = workspace(d), offsets_of(counts, first)
    for accumulate in (False, True):
        before = db.double().clone()
        G.goldy_linear_bias_grad(d, ptr(dy), ptr(db), z=ptr(z), dz=ptr(dz), accumulate=accumulate, offsets=ptr(off),
                                 workspace=ptr(ws), workspace_bytes=ws.numel(),
                                 stream=torch.cuda.current_stream().cuda_stream)
        finish(ws)
        for e, lo, hi in spans(rows, counts, first):
            g = dy[lo:hi].double()
            if act != "none":
                z64 = z[lo:hi].double()
                err = 1e-6 * (1 + z64.abs()) * g.abs()
                g = g * slope64(z64, act)
                if hi > lo:
                    check(dz[lo:hi], g, err + round_tol(g, BF16) * 1.01, f"dZ of group {e}")
            ref = g.sum(0) + (before[e] if accumulate else 0)
            # every term passes at most rows / (8 warps * slices) + 8 + slices additions
            bound = (hi - lo + 20) * 2.0 ** -24 * (g.abs().sum(0) + (before[e].abs() if accumulate else 0))
            if act != "none":
                bound = bound + err.sum(0)
            check(db[e], ref, bound + 1e-30, f"db of group {e}")


def test_gradients_against_differences(cuda_ok):
    """dX, dW and db of act(X W + b) against central differences of the fp64
    forward pass along random directions (third-order error of the difference:
    h^2 times the third derivative; rounding of the bf16 dZ and dX: 2^-8 of
    each term, far below the 1% bound after summing thousands of terms)."""
    rows, k, n, act = 120, 96, 160, "gelu"
    gen = gen_of(8)
    x, w = matrix(gen, rows, k), matrix(gen, k, n, None, k ** -0.5)
    b = torch.randn(n, generator=gen, device="cuda").bfloat16()
    g = matrix(gen, rows, n)
    z, y = out_matrix(rows, n, BF16), out_matrix(rows, n, BF16)
    d = G.linear_desc(rows, k, n, act=ACTS[act])
    ws = workspace(d)
    kw = dict(workspace=ptr(ws), workspace_bytes=ws.numel(), stream=torch.cuda.current_stream().cuda_stream)
    G.goldy_linear_forward(d, ptr(x), ptr(w), ptr(y), bias=ptr(b), z=ptr(z), **kw)
    dz, dx = torch.empty_like(g), out_matrix(rows, k, BF16)
    dw, db = out_matrix(k, n, F32), torch.empty(n, device="cuda")
    G.goldy_linear_bias_grad(d, ptr(g), ptr(db), z=ptr(z), dz=ptr(dz), **kw)
    G.goldy_linear_input_grad(d, ptr(dz), ptr(w), ptr(dx), **kw)
    G.goldy_linear_weight_grad(d, ptr(x), ptr(dz), ptr(dw), **kw)
    finish(ws)
    loss = lambda x, w, b: float((act64(x @ w + b, act) * g.double()).sum())  # noqa: E731
    at = [t.double() for t in (x, w, b)]
    h = 1e-4
    for i, grad in enumerate((dx, dw, db)):
        v = grad.double() / grad.double().norm()          # along the gradient: the slope is its norm
        lo, hi = list(at), list(at)
        lo[i], hi[i] = at[i] - h * v, at[i] + h * v
        slope = (loss(*hi) - loss(*lo)) / (2 * h)
        assert abs(slope - float((grad.double() * v).sum())) < 0.01 * abs(slope)


def test_empty_sizes(cuda_ok):
    run_forward(0, 64, 64)
    run_forward(64, 64, 0, bias=False, ldw=8, ldy=8)
    y = run_forward(37, 0, 100, act="gelu", residual=True)          # act(b) + R
    assert torch.isfinite(y[:37].float()).all()
    run_weight_grad(0, 72, 40)
    run_weight_grad(0, 72, 40, accumulate=True)
    run_weight_grad(0, 72, 40, counts=[0, 0, 0])
    run_input_grad(21, 80, 0)


def test_results_do_not_depend_on_the_run(cuda_ok):
    """The same bits every time, on any stream, eagerly or from a graph."""
    rows, k, n = 37, 4096, 1024                                      # a split reduction
    gen = gen_of(2)
    x, w = matrix(gen, rows, k), matrix(gen, k, n, None, k ** -0.5)
    d = G.linear_desc(rows, k, n)
    ws = workspace(d)
    ys = [out_matrix(rows, n, BF16) for _ in range(4)]

    def go(y, stream):
        G.goldy_linear_forward(d, ptr(x), ptr(w), ptr(y), workspace=ptr(ws), workspace_bytes=ws.numel(), stream=stream.cuda_stream)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    go(ys[0], s)
    go(ys[1], s)
    s.synchronize()
    go(ys[2], torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        go(ys[3], s)
    graph.replay()
    graph.replay()
    finish(ws)
    for y in ys[1:]:
        assert torch.equal(ys[0], y)


def test_order_on_a_stream(cuda_ok):
    """Offsets, inputs and residuals written by earlier work of the stream are
    seen, back to back and without synchronisation."""
    rows, k, n = 300, 256, 384
    gen = gen_of(5)
    x, w = matrix(gen, rows, k), matrix(gen, k, k, None, k ** -0.5)
    d = G.linear_desc(rows, k, k)
    ws = workspace(d)
    bufs = [x.clone()] + [out_matrix(rows, k, BF16) for _ in range(12)]
    s = torch.cuda.current_stream().cuda_stream
    for a, b in zip(bufs, bufs[1:]):
        G.goldy_linear_forward(d, ptr(a), ptr(w), ptr(b), workspace=ptr(ws), workspace_bytes=ws.numel(), stream=s)
    finish(ws)
    for a, b in zip(bufs, bufs[1:]):
        ref, sab = a.double() @ w.double(), a.double().abs() @ w.double().abs()
        check(b, ref, (k / 16 + 2) * 2.0 ** -22 * sab + round_tol(ref, BF16) * 1.01, "chained product")


def test_residual_in_place(cuda_ok):
    rows, k, n = 90, 128, 200
    gen = gen_of(6)
    x, w = matrix(gen, rows, k), matrix(gen, k, n, None, k ** -0.5)
    y = torch.randn(rows, n, generator=gen, device="cuda")
    before = y.double().clone()
    d = G.linear_desc(rows, k, n, y_dtype=F32)
    ws = workspace(d)
    G.goldy_linear_forward(d, ptr(x), ptr(w), ptr(y), residual=ptr(y), workspace=ptr(ws), workspace_bytes=ws.numel(),
                           stream=torch.cuda.current_stream().cuda_stream)
    finish(ws)
    ref, s = x.double() @ w.double() + before, x.double().abs() @ w.double().abs() + before.abs()
    check(y, ref, (steps(k, F32) + 3) * 2.0 ** -22 * s, "Y += X W")


def test_offsets_past_32_bits(cuda_ok):
    """Row strides whose byte offsets need more than 32 bits."""
    rows, k, n = 5, 72, 72
    gen = gen_of(9)
    ld = 1 << 29                                                     # 5 rows of 1 GiB
    x = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)[:, :k]
    x.copy_(torch.randn(rows, k, generator=gen, device="cuda"))
    w = matrix(gen, k, n, None, k ** -0.5)
    y = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)[:, :n]
    d = G.linear_desc(rows, k, n, ldx=ld, ldy=ld)
    ws = workspace(d)
    G.goldy_linear_forward(d, ptr(x), ptr(w), ptr(y), workspace=ptr(ws), workspace_bytes=ws.numel(),
                           stream=torch.cuda.current_stream().cuda_stream)
    finish(ws)
    ref, s = x.double() @ w.double(), x.double().abs() @ w.double().abs()
    check(y, ref, (k / 16 + 2) * 2.0 ** -22 * s + round_tol(ref, BF16) * 1.01, "Y with a long stride")


def test_offsets_that_are_not_ordered(cuda_ok):
    """Decreasing or out-of-range offsets touch nothing outside the arrays."""
    rows, k, n = 100, 64, 128
    gen = gen_of(10)
    x, w = matrix(gen, rows, k), matrix(gen, k, n, None, k ** -0.5, (4,))
    y = torch.full((rows + 64, n), 7.0, device="cuda", dtype=torch.bfloat16)
    off = torch.tensor([-5, 80, 20, 1 << 30, 60], dtype=torch.int32, device="cuda")
    d = G.linear_desc(rows, k, n, groups=4)
    ws = workspace(d)
    dw, db = torch.empty(4, k, n, device="cuda"), torch.empty(4, n, device="cuda")
    kw = dict(offsets=ptr(off), workspace=ptr(ws), workspace_bytes=ws.numel(), stream=torch.cuda.current_stream().cuda_stream)
    G.goldy_linear_forward(d, ptr(x), ptr(w), ptr(y), **kw)
    G.goldy_linear_weight_grad(d, ptr(x), ptr(y), ptr(dw), **kw)
    G.goldy_linear_bias_grad(d, ptr(y), ptr(db), **kw)
    finish(ws)
    assert (y[rows:] == 7.0).all()


def test_in_an_sm_partition(cuda_ok):
    """On a partition's stream the calls run inside it, with the same results."""
    rows, k, n, counts = 300, 512, 640, [100, 0, 37, 163]
    gen = gen_of(12)
    x, w, dy = matrix(gen, rows, k), matrix(gen, k, n, None, k ** -0.5, (4,)), matrix(gen, rows, n)
    off = offsets_of(counts)
    d = G.linear_desc(rows, k, n, groups=4, dw_dtype=F32)
    ws = workspace(d)
    part = G.goldy_partition_create(16, 1)
    sms, streams = G.goldy_partition_query(part, 1)
    assert 16 <= sms < 152
    results = []
    for stream in (torch.cuda.current_stream().cuda_stream, streams[0]):
        y, dw, db = out_matrix(rows, n, BF16), out_matrix(k, n, F32, lead=(4,)), torch.empty(4, n, device="cuda")
        torch.cuda.synchronize()
        kw = dict(offsets=ptr(off), workspace=ptr(ws), workspace_bytes=ws.numel(), stream=stream)
        G.goldy_linear_forward(d, ptr(x), ptr(w), ptr(y), **kw)
        G.goldy_linear_weight_grad(d, ptr(x), ptr(dy), ptr(dw), **kw)
        G.goldy_linear_bias_grad(d, ptr(dy), ptr(db), **kw)
        finish(ws)
        results.append((y, dw, db))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    part.close()
