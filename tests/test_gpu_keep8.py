"""Rows kept in 8 bits against the definition, bit by bit, and what is read back.

H is the layer operators' activation of the value that was kept.  Its error, before
the rounding to the rows' type: relu and none none; silu and gelu by tanh are z
times a sigmoid of v (v = z, or 1.6 (z + 0.045 z^3), computed to 4 u): the exponent
is off by 5 |v| u, the exponential, the reciprocal, the sum and the product by 8 u
together, so (5 |v| + 8) u of the result (v beyond 90: below 1e-36, absolutely);
gelu by 7.1.26 of Abramowitz and Stegun: |z| (1.5e-7 + 8 u)."""
import math

import pytest
import torch

from expert_ops_util import HALF, TYPES, U, Rows, act64, gen_of, within
from paper_2409_02227_gb300 import goldy as G

pytestmark = pytest.mark.gpu
ACTS = [G.GOLDY_ACT_NONE, G.GOLDY_ACT_RELU, G.GOLDY_ACT_GELU, G.GOLDY_ACT_GELU_TANH, G.GOLDY_ACT_SILU]
BLOCK = G.GOLDY_KEEP8_BLOCK
# the value of every e4m3 byte
E4M3 = [(-1.0) ** (b >> 7) * ((b & 7) / 8 * 2.0 ** -6 if (b >> 3 & 15) == 0 else (1 + (b & 7) / 8) * 2.0 ** ((b >> 3 & 15) - 7))
        for b in range(256)]


def kept_plainly(z):
    """(bytes, scale bytes) by a search over powers and a table of values, in fp64 on the CPU."""
    z = z.double().cpu()
    rows, n = z.shape
    blocks = -(-n // BLOCK)
    z = torch.cat([z, torch.zeros(rows, blocks * BLOCK - n, dtype=torch.float64)], 1).view(rows, blocks, BLOCK)
    finite = torch.where(torch.isfinite(z), z.abs(), 0.0).amax(2)
    e = torch.full((rows, blocks), -127, dtype=torch.int64)
    while bool((over := finite > 448 * torch.pow(torch.tensor(2.0, dtype=torch.float64), e)).any()):
        e[over] += 1
    v = z / torch.pow(torch.tensor(2.0, dtype=torch.float64), e)[:, :, None]
    table = torch.tensor(E4M3[:127], dtype=torch.float64)
    up = torch.searchsorted(table, v.abs().nan_to_num(0.0, 0.0, 0.0).contiguous()).clamp(max=126)
    low = (up - 1).clamp(min=0)
    a = v.abs().nan_to_num(0.0, 0.0, 0.0)
    to_up, to_low = table[up] - a, a - table[low]
    code = torch.where((to_up < to_low) | ((to_up == to_low) & (up % 2 == 0)), up, low)
    code = code + 128 * (torch.signbit(v))
    code = torch.where(torch.isfinite(z), code, 127)
    return code.to(torch.uint8).view(rows, -1), (e + 127).to(torch.uint8)


def pack(rows_, d):
    q_bytes, s_bytes = G.goldy_keep8_query(d)
    q = torch.full((q_bytes + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    s = torch.full((s_bytes + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    G.goldy_keep8_pack(d, rows_.ptr, q.data_ptr(), s.data_ptr())
    torch.cuda.synchronize()
    assert (q[q_bytes:] == 0xA5).all() and (s[s_bytes:] == 0xA5).all()
    return q[:q_bytes].view(d.rows, -1), s[:s_bytes].view(d.rows, -1)


def spread(gen, rows, n):
    """Values over many powers of two, blocks of different size, some zero."""
    z = torch.randn(rows, n, generator=gen, device="cuda") * torch.exp2(torch.randint(-9, 3, (rows, n), generator=gen, device="cuda"))
    z = z * torch.exp2(torch.randint(-30, 31, (1, n), generator=gen, device="cuda")).float()
    z[torch.rand(rows, n, generator=gen, device="cuda") < 0.05] = 0.0
    return z


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n,more,start", [(1, 1, 0, 0), (2, 31, 0, 0), (3, 32, 0, 0), (5, 33, 0, 1), (7, 100, 4, 0),
                                               (64, 264, 8, 8), (9, 1000, 0, 0), (9, 1001, 2, 3), (3, 4096, 0, 0),
                                               (2, 20011, 5, 7), (3000, 40, 0, 0)])
def test_pack_and_unpack(cuda_ok, rows, n, more, start, dtype):
    t = TYPES[dtype][0]
    z = Rows(rows, n, t, n + more, start, spread(gen_of(n), rows, n))
    d = G.keep8_desc(rows, n, dtype=TYPES[dtype][1], ldz=n + more, ldh=n + 3)
    q, s = pack(z, d)
    want_q, want_s = kept_plainly(z.t)
    assert torch.equal(s.cpu(), want_s)
    # -0 where a negative number is rounded to 0 is as good as 0
    same = (q.cpu() == want_q) | ((q.cpu() & 127) == 0) & ((want_q & 127) == 0)
    assert same.all()
    assert (q.cpu()[:, n:] == 0).all()
    back, h = Rows(rows, n, t, n + more, start), Rows(rows, n, t, n + 3, 1)
    G.goldy_keep8_unpack(d, q.data_ptr(), s.data_ptr(), back.ptr, h.ptr)
    torch.cuda.synchronize()
    value = torch.tensor(E4M3, dtype=torch.float64)[want_q.long()].view(rows, -1, BLOCK)
    value = (value * torch.pow(torch.tensor(2.0, dtype=torch.float64), want_s.double() - 127)[:, :, None]).view(rows, -1)[:, :n]
    assert torch.equal(back.t.double().cpu(), value)        # nothing here underflows: e >= -50
    assert torch.equal(h.t, back.t) and back.guarded() and h.guarded()
    # the definition's error
    far = (value - z.t.double().cpu()).abs()
    step = torch.pow(torch.tensor(2.0, dtype=torch.float64), want_s.double() - 127 - 10).repeat_interleave(BLOCK, 1)[:, :n]
    assert (far <= torch.maximum(z.t.double().cpu().abs() / 16, step)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_act(cuda_ok, act, dtype):
    rows, n, t = 64, 1000, TYPES[dtype][0]
    z = 3.0 * torch.randn(rows, n, generator=gen_of(act), device="cuda")
    z[0], z[1, :500], z[1, 500:] = 0.0, 60.0, -60.0
    z[2] = torch.linspace(-12, 12, n, device="cuda")
    z = Rows(rows, n, t, fill=z)
    d = G.keep8_desc(rows, n, dtype=TYPES[dtype][1], act=act)
    q, s = pack(z, d)
    back, h, h2 = Rows(rows, n, t), Rows(rows, n, t), Rows(rows, n, t)
    G.goldy_keep8_unpack(d, q.data_ptr(), s.data_ptr(), back.ptr, h.ptr)
    G.goldy_keep8_unpack(d, q.data_ptr(), s.data_ptr(), 0, h2.ptr)
    torch.cuda.synchronize()
    v = back.t.double()
    ref = act64(v, act)
    if act in (G.GOLDY_ACT_NONE, G.GOLDY_ACT_RELU):
        tol = torch.zeros_like(ref)
    elif act == G.GOLDY_ACT_GELU:
        tol = v.abs() * (1.5e-7 + 8 * U)
    else:
        arg = v.abs() if act == G.GOLDY_ACT_SILU else 1.6 * (v.abs() + 0.045 * v.abs() ** 3)
        tol = (5 * arg + 8) * U * ref.abs() + 1e-36
    within(h.t, ref, tol + HALF[t] * ref.abs(), "H")
    assert torch.equal(h.t, h2.t)


def test_far_apart(cuda_ok):
    """Rows of Z and H more than 2^32 elements apart."""
    rows, n, ld = 70000, 40, 70000
    z = Rows(rows, n, torch.bfloat16, ld, 0, torch.randn(rows, n, generator=gen_of(1), device="cuda"))
    packed = z.t.contiguous()
    d, dense = G.keep8_desc(rows, n, ldz=ld, ldh=ld, act=G.GOLDY_ACT_SILU), G.keep8_desc(rows, n, act=G.GOLDY_ACT_SILU)
    q_bytes, s_bytes = G.goldy_keep8_query(d)
    (q, s), (q2, s2) = ([torch.zeros(b, dtype=torch.uint8, device="cuda") for b in (q_bytes, s_bytes)] for _ in range(2))
    G.goldy_keep8_pack(d, z.ptr, q.data_ptr(), s.data_ptr())
    G.goldy_keep8_pack(dense, packed.data_ptr(), q2.data_ptr(), s2.data_ptr())
    h, z2, h2 = Rows(rows, n, torch.bfloat16, ld), torch.empty_like(packed), torch.empty_like(packed)
    G.goldy_keep8_unpack(d, q.data_ptr(), s.data_ptr(), z.ptr, h.ptr)
    G.goldy_keep8_unpack(dense, q2.data_ptr(), s2.data_ptr(), z2.data_ptr(), h2.data_ptr())
    torch.cuda.synchronize()
    assert torch.equal(q, q2) and torch.equal(s, s2) and torch.equal(z.t, z2) and torch.equal(h.t, h2)


def test_edges(cuda_ok):
    """The largest value at, just below and just above 448 powers; ties; zeros;
    the smallest and largest numbers."""
    rows = torch.zeros(8, 64)
    rows[0, :4] = torch.tensor([448.0, 449.0, 28.5, -26.0])          # 449: the next power
    rows[0, 32:35] = torch.tensor([448.0, 17.0, -19.0])
    rows[1, :6] = torch.tensor([1.0, 1.0625, 1.1875, -1.0625, -1.1875, 1.3125])
    rows[1, 32:36] = torch.tensor([1.75, 2 ** -13.0, 3 * 2 ** -18.0, 2 ** -18.0])
    rows[2, 0], rows[2, 32] = 3.0e38, -3.4028234663852886e38
    rows[3, 0], rows[3, 1], rows[3, 32] = 1e-38, 1e-40, 1.4e-45
    rows[4, 63] = -2.0
    rows[5, :3] = torch.tensor([math.inf, 5.0, -7.0])
    rows[5, 32:35] = torch.tensor([math.nan, -math.inf, 0.0])
    rows[6] = -math.inf
    z = Rows(8, 64, torch.float32, fill=rows)
    d = G.keep8_desc(8, 64, dtype=G.GOLDY_F32)
    q, s = pack(z, d)
    want_q, want_s = kept_plainly(z.t)
    assert torch.equal(s.cpu(), want_s)
    assert ((q.cpu() == want_q) | ((q.cpu() & 127) == 0) & ((want_q & 127) == 0) | ((q.cpu() & 127) == 127) & (want_q == 127)).all()
    back = Rows(8, 64, torch.float32)
    G.goldy_keep8_unpack(d, q.data_ptr(), s.data_ptr(), back.ptr)
    torch.cuda.synchronize()
    assert torch.equal(torch.isnan(back.t).cpu(), ~torch.isfinite(rows))
    assert back.t[5, 1] == 5.0 and back.t[5, 2] == -7.0
    assert float(back.t[2, 0]) == 3.0e38 / 1.0 or abs(float(back.t[2, 0]) / 3.0e38 - 1) <= 2 ** -4
