"""The workspace: exactly the queried bytes are enough, nothing behind them is
written, what an earlier call left in it (NaN here) does not matter, and a smaller
one is refused."""
import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from test_gpu_linear import ACTS, F32, NAN, gen_of, offsets_of, ptr

pytestmark = pytest.mark.gpu

GUARD = 1 << 20


def used(need):
    """`need` bytes, counters zero, the rest NaN, and a patterned guard behind."""
    ws = torch.zeros((need + 255) // 256 * 256 + GUARD, dtype=torch.uint8, device="cuda")
    ws[65536:need // 4 * 4].view(torch.float32).fill_(NAN)
    ws[need:] = 0xA5
    return ws


def intact(ws, need):
    torch.cuda.synchronize()
    assert (ws[need:] == 0xA5).all(), "written behind the workspace"
    assert not ws[:65536].any(), "counters are not zero after the call"


# splits of the reduction, operands' copies, many experts, long reductions
@pytest.mark.parametrize("rows,k,n,counts,pad", [(1, 4096, 512, None, 0), (37, 4096, 1024, None, 0), (50, 75, 130, None, 0),
                                                 (37, 4097, 1023, None, 0), (300, 131, 259, [100, 0, 37, 163], 0),
                                                 (64, 1024, 256, [1] * 60 + [0, 4], 0), (2000, 72, 65, [3] * 500, 1),
                                                 (70001, 130, 200, None, 0), (600, 2048, 128, [600], 0)])
@pytest.mark.parametrize("out", [G.GOLDY_BF16, F32])
def test_linear(cuda_ok, rows, k, n, counts, pad, out):
    gen, groups = gen_of(rows + k), len(counts or [])
    lead = (groups,) if groups else ()
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    x, w, dy, z = rnd(rows, k + pad), rnd(*lead, k, n), rnd(rows, n), rnd(rows, n)
    kind = torch.bfloat16 if out == G.GOLDY_BF16 else torch.float32
    d = G.linear_desc(rows, k, n, groups=groups, act=ACTS["gelu"], y_dtype=out, dx_dtype=out, dw_dtype=out, ldx=k + pad,
                      lddx=k, ldw=n, ldy=n, ldz=n)
    off, need = offsets_of(counts), G.goldy_linear_query(d)
    assert need > 65536
    results, refused = [], 0
    for size, ws in ((need, used(need)), (1 << 30, torch.zeros(1 << 30, dtype=torch.uint8, device="cuda")),
                     (need - 1, used(need))):
        y, dx = torch.full((rows, n), NAN, device="cuda", dtype=kind), torch.full((rows, k), NAN, device="cuda", dtype=kind)
        dw, db = torch.full((*lead, k, n), NAN, device="cuda", dtype=kind), torch.full((*lead, n), NAN, device="cuda")
        dz = torch.full_like(dy, NAN)
        kw = dict(offsets=ptr(off), workspace=ptr(ws), workspace_bytes=size, stream=torch.cuda.current_stream().cuda_stream)
        for call in (lambda: G.goldy_linear_forward(d, ptr(x), ptr(w), ptr(y), **kw),
                     lambda: G.goldy_linear_input_grad(d, ptr(dy), ptr(w), ptr(dx), **kw),
                     lambda: G.goldy_linear_weight_grad(d, ptr(x), ptr(dy), ptr(dw), **kw),
                     lambda: G.goldy_linear_bias_grad(d, ptr(dy), ptr(db), z=ptr(z), dz=ptr(dz), **kw)):
            try:
                call()
            except G.GoldyError as e:
                assert size == need - 1 and e.status == G.GOLDY_ERR_NOMEM
                refused += 1
            if size != 1 << 30:
                intact(ws, need)
        results.append((y, dx, dw, db, dz))
    assert refused >= 1, "no call needs what the query asks for"
    live = sum(counts) if counts else rows                  # the rest are no expert's: not written
    for i, (a, b) in enumerate(zip(*results[:2])):
        a, b = (a[:live], b[:live]) if i in (0, 1, 4) else (a, b)
        assert torch.equal(a, b)
        assert torch.isfinite(a.float()).all()
    assert G.goldy_device_error(clear=True) == 0


@pytest.mark.parametrize("rows,n", [(0, 100), (1, 30), (7, 1000), (3000, 1023), (400, 4096), (200, 9000), (3, 60000), (160, 70000)])
@pytest.mark.parametrize("dtype", [G.GOLDY_BF16, F32])
def test_layernorm(cuda_ok, rows, n, dtype):
    gen = gen_of(n)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    kind = torch.bfloat16 if dtype == G.GOLDY_BF16 else torch.float32
    x, dy, mean, rstd = rnd(rows, n).to(kind), rnd(rows, n).to(kind), rnd(rows), 1 + rnd(rows).abs()
    d = G.layernorm_desc(rows, n, dtype=dtype, param_dtype=F32)
    need, results = G.goldy_layernorm_query(d), []
    for size, ws in ((need, used(need)), (1 << 30, torch.zeros(1 << 30, dtype=torch.uint8, device="cuda"))):
        dx, dg, db = torch.full((rows, n), NAN, device="cuda", dtype=kind), *torch.full((2, n), NAN, device="cuda")
        G.goldy_layernorm_backward(d, ptr(dy), ptr(x), 0, ptr(mean), ptr(rstd), ptr(dx), ptr(dg), ptr(db), ptr(ws), size,
                                   torch.cuda.current_stream().cuda_stream)
        if size == need:
            intact(ws, need)
        torch.cuda.synchronize()
        results.append((dx, dg, db))
    for a, b in zip(*results):
        assert torch.isfinite(a.float()).all() and torch.equal(a, b)
    with pytest.raises(G.GoldyError) as e:
        G.goldy_layernorm_backward(d, ptr(dy), ptr(x), 0, ptr(mean), ptr(rstd), ptr(dx), ptr(dg), ptr(db), ptr(ws), need - 1,
                                   torch.cuda.current_stream().cuda_stream)
    assert e.value.status == G.GOLDY_ERR_NOMEM
