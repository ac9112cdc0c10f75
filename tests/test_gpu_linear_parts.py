"""fp32 results at reductions around and beyond the parts that are added up, with
the bound that follows from the kernel's rule: a reduction of ceil(K / 64) stages is
cut into equal parts of at most 12, within which the tensor cores truncate 4 times a
stage (2^-22 of the sum of absolute terms at most), and the parts, and at most 8
splits of the reduction, are added with rounding to nearest."""
import math

import pytest

import test_gpu_linear as base
from test_gpu_linear import BF16, F32

pytestmark = pytest.mark.gpu


def steps(k, dtype):
    if dtype == BF16:
        return k / 16
    stages = math.ceil(k / 64)
    parts = max(1, math.ceil(stages / 12))
    return 4 * math.ceil(stages / parts) + (parts + 8) / 4        # an addition: 2^-24


@pytest.mark.parametrize("k", [512, 700, 768, 769, 832, 1500, 1536, 1537, 2048, 5000, 8192, 16384])
@pytest.mark.parametrize("rows,n", [(3, 72), (200, 136), (500, 1024)])
def test_long_reductions(cuda_ok, monkeypatch, k, rows, n):
    monkeypatch.setattr(base, "steps", steps)
    base.run_forward(rows, k, n, y_dtype=F32, seed=k)
    base.run_input_grad(rows, n, k, dx_dtype=F32, seed=k)
    base.run_weight_grad(k, n, rows, dw_dtype=F32, seed=k)
    base.run_weight_grad(k, n, rows, dw_dtype=F32, accumulate=True, seed=k)
