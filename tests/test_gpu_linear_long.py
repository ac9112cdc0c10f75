"""Weight gradients in bf16 over very many rows.

All terms are positive here, so that an accumulator that truncates is off to one
side.  Rounding to bf16 is off by at most half a unit in the last place of the
result.  Before it, a sum of parts of at most 8192 rows may be off by 512 steps of
2^-22 within a part (the tensor cores' truncation) and by 2^-24 for each of
the additions, rounded to nearest, that join the parts: rows / 4096 + 16 of them
(equal parts of more than half the limit, splits, the sum that it is added to).
That is 1.6e-4 or less of the result here; one accumulator loses 1e-9 per row,
1e-3 and more.
"""
import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from test_gpu_linear import BF16, finish, gen_of, offsets_of, out_matrix, ptr, spans, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,k,n,counts,first,accumulate", [(3_000_000, 64, 136, None, 0, False),
                                                              (1_000_003, 200, 264, None, 0, True),
                                                              (2_500_000, 72, 128, [2_000_000, 0, 499_001], 900, False)])
def test_bf16_weight_gradient_over_many_rows(cuda_ok, rows, k, n, counts, first, accumulate):
    gen, lead = gen_of(rows), (len(counts),) if counts else ()
    # columns of different sizes, so that the results' roundings differ
    scale = lambda c: torch.exp(torch.randn(c, generator=gen, device="cuda"))  # noqa: E731
    x = (torch.rand(rows, k, generator=gen, device="cuda") * scale(k)).bfloat16()
    dy = (torch.rand(rows, n, generator=gen, device="cuda") * scale(n)).bfloat16()
    dw = out_matrix(k, n, BF16, lead=lead)
    if accumulate:
        dw[...] = (rows * torch.rand(k, n, generator=gen, device="cuda")).bfloat16()
    before = dw.double().clone()
    d = G.linear_desc(rows, k, n, groups=len(counts or []), dw_dtype=BF16, ldw=n, ldx=k, ldy=n)
    ws, off = workspace(d), offsets_of(counts, first)
    G.goldy_linear_weight_grad(d, ptr(x), ptr(dy), ptr(dw), accumulate=accumulate, offsets=ptr(off), workspace=ptr(ws),
                               workspace_bytes=ws.numel(), stream=torch.cuda.current_stream().cuda_stream)
    finish(ws)
    for e, lo, hi in spans(rows, counts, first):
        ref = sum((x[i:min(i + 250_000, hi)].double().T @ dy[i:min(i + 250_000, hi)].double()
                   for i in range(lo, hi, 250_000)), torch.zeros(k, n, device="cuda", dtype=torch.float64))
        got = (dw[e] if counts else dw).double()
        tol = (512 * 2.0 ** -22 + ((hi - lo) / 4096 + 16) * 2.0 ** -24) * ref
        if accumulate:
            ref = ref + before
        tol = tol + torch.exp2(torch.floor(torch.log2(ref.clamp(min=1e-30) + tol)) - 8)   # half a unit, 8 significant bits
        assert torch.isfinite(got).all()
        over = (got - ref).abs() - tol
        assert not (over > 0).any(), f"dW of group {e}: {int((over > 0).sum())} of {over.numel()} beyond their bound"
