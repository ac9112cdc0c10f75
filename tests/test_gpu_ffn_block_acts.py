"""The feed-forward block with each activation, none included, against automatic
differentiation in fp64 (bound: test_gpu_ffn_block.py).

That bound takes slopes that change little when the normed rows are rounded to
bf16.  relu's jumps from 0 to 1 at 0: rounding moves about one pre-activation
in a thousand across (a share s of wrong slopes is sqrt(s) of a gradient's norm, 3e-2).
Such a value's slope may be either, so relu's reference takes the sign of the
pre-activations that the block has saved.
"""
import math

import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from paper_2409_02227_gb300.ffn_block import FeedForward
from test_gpu_ffn_block import near
from test_gpu_linear import ACTS, act64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", list(ACTS))
def test_activation(cuda_ok, act):
    rows, width, hidden = 130, 128, 264
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    block = FeedForward(rows, width, hidden, act=ACTS[act], seed=1)
    x, dy = (torch.randn(rows, width, generator=gen, device="cuda").bfloat16() for _ in range(2))
    y = block.forward(x)
    dx = block.backward(dy)
    torch.cuda.synchronize()
    assert G.goldy_device_error(clear=True) == 0
    p = {k: v.double().clone().requires_grad_(True) for k, v in block.p.items()}
    x64 = x.double().requires_grad_(True)
    c = x64 - x64.mean(1, keepdim=True)
    n = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * p["gamma"] + p["beta"]
    assert math.isclose(block.norm.eps, 1e-5, rel_tol=1e-6)
    z = n @ p["w1"] + p["b1"]
    h = z * (block.z > 0) if act == "relu" else act64(z, act)
    ref = x64 + h @ p["w2"] + p["b2"]
    ref.backward(dy.double())
    near(y, ref.detach(), "y")
    near(dx, x64.grad, "dx")
    for k, v in p.items():
        near(block.grads[k], v.grad, k)
