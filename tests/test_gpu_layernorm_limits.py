"""Layer norm at the largest row length: indices of a partial row, 2 n of them,
pass 31 bits."""
import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from test_gpu_layernorm import BF16, NAN, ptr, stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [(1 << 30) - 1, 1 << 30])
def test_no_rows_of_the_largest_length(cuda_ok, n):
    d = G.layernorm_desc(0, n, dtype=BF16)
    ws = torch.zeros(G.goldy_layernorm_query(d), dtype=torch.uint8, device="cuda")
    ws[65536:].view(torch.float32).fill_(NAN)
    dg, db = torch.full((n,), NAN, device="cuda"), torch.full((n,), NAN, device="cuda")
    G.goldy_layernorm_backward(d, 0, 0, 0, 0, 0, 0, ptr(dg), ptr(db), ptr(ws), ws.numel(), stream())
    torch.cuda.synchronize()
    assert not dg.any() and not db.any()
    assert not ws[:65536].any()
