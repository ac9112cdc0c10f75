"""The feed-forward block against automatic differentiation in fp64 on the
same bf16 weights and inputs.

Bound: the block rounds to bf16 (2^-8 of an element, 1.7e-3 of a tensor's norm)
the normed input, the pre-activation's copy, the hidden rows, dZ, the norm's
incoming gradient and its results; each rounding reaches a result at most once
with gain about 1, so six of them stay below 1.5e-2 of its norm."""
import math

import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from paper_2409_02227_gb300.ffn_block import FeedForward

pytestmark = pytest.mark.gpu


def reference(block, x, ids, dy):
    p = {k: v.double().clone().requires_grad_(True) for k, v in block.p.items()}
    x = x.double().clone().requires_grad_(True)
    mean = x.mean(1, keepdim=True)
    n = (x - mean) / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + 1e-5) * p["gamma"] + p["beta"]
    gelu = lambda z: 0.5 * z * torch.erfc(-z / math.sqrt(2))  # noqa: E731
    if ids is None:
        y = x + gelu(n @ p["w1"] + p["b1"]) @ p["w2"] + p["b2"]
    else:
        y = x
        for e in range(block.experts):
            at = (ids == e).nonzero()[:, 0]
            if len(at):
                out = gelu(n[at] @ p["w1"][e] + p["b1"][e]) @ p["w2"][e] + p["b2"][e]
                y = y.index_add(0, at, out)
    y.backward(dy.double())
    return y.detach(), x.grad, {k: v.grad if v.grad is not None else torch.zeros_like(v) for k, v in p.items()}


def near(got, ref, what):
    assert torch.isfinite(got).all(), what
    off = float((got.double() - ref).norm() / ref.norm())
    assert off < 1.5e-2, f"{what}: {off:.2e}"


@pytest.mark.parametrize("rows,width,hidden,experts", [(100, 136, 264, 0), (513, 512, 1024, 0), (300, 128, 512, 5),
                                                       (64, 256, 256, 40)])
def test_block(cuda_ok, rows, width, hidden, experts):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows)
    block = FeedForward(rows, width, hidden, experts, seed=1)
    x = torch.randn(rows, width, generator=gen, device="cuda").bfloat16()
    dy = torch.randn(rows, width, generator=gen, device="cuda").bfloat16()
    ids = None
    if experts:
        ids = torch.randint(0, experts, (rows,), generator=gen, device="cuda")
        ids[ids == 1] = 0                                   # an expert without rows
        for k in ("b1", "b2"):
            block.p[k].normal_(generator=gen)
    y = block.forward(x, ids)
    dx = block.backward(dy)
    torch.cuda.synchronize()
    assert G.goldy_device_error(clear=True) == 0
    ry, rdx, rg = reference(block, x, ids, dy)
    near(y, ry, "y")
    near(dx, rdx, "dx")
    for k, ref in rg.items():
        near(block.grads[k], ref, k)
    if experts:
        assert (block.grads["w1"][1] == 0).all() and (block.grads["b2"][1] == 0).all()


def test_descent(cuda_ok):
    """Steps below 2 / (largest curvature) lower the loss every time.  The
    loss is the mean over rows of a squared norm; its curvature in W2 is at
    most 2 |hidden row|^2, about 2 * 512 * 0.4 here, and of the same order in
    the other weights, so 2e-4 is safe by an order of magnitude."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    x = torch.randn(256, 128, generator=gen, device="cuda").bfloat16()
    target = torch.randn(256, 128, generator=gen, device="cuda")
    block = FeedForward(256, 128, 512)
    losses = []
    for _ in range(6):
        error = block.forward(x).float() - target
        losses.append(float(error.square().sum(1).mean()))
        block.backward((error * (2.0 / 256)).bfloat16())
        block.step(2e-4)
    assert all(b < a for a, b in zip(losses, losses[1:])), losses
