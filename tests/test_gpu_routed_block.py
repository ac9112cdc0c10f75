"""The routed feed-forward block against automatic differentiation in fp64 with the
experts that it chose.

Bound.  As for the plain block a rounding to bf16 is 1.7e-3 of a tensor's norm; here
the normed input, the hidden rows, the experts' rows, their sum, dF, the experts'
gradient, dZ, the rows' gradient, their sum and the norm's gradient are rounded,
and a result lies behind twelve of those at most: 2e-2.  The router's gradient is
a difference of terms about as large as itself, after six roundings: 3e-2.  Kept
in 8 bits, a pre-activation is off by up to 2^-4, 2.6e-2 of its norm (evenly
spread up to half a step of 2^-3 to 2^-4); the hidden rows and the activation's
slope take that over, at most with gain 1.5 each: 8e-2 more for what the backward
pass makes from them."""
import math

import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from paper_2409_02227_gb300.ffn_block import RoutedFeedForward

pytestmark = pytest.mark.gpu
ACT64 = {G.GOLDY_ACT_GELU: lambda z: 0.5 * z * torch.erfc(-z / math.sqrt(2)), G.GOLDY_ACT_SILU: lambda z: z / (1 + torch.exp(-z)),
         G.GOLDY_ACT_NONE: lambda z: z}


def reference(block, x, dy, act, post, alpha, over):
    p = {k: v.double().clone().requires_grad_(True) for k, v in block.p.items()}
    x = x.double().clone().requires_grad_(True)
    mean = x.mean(1, keepdim=True)
    n = (x - mean) / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + 1e-5) * p["gamma"] + p["beta"]
    ids = block.ids.long()
    logits = n @ p["wr"]
    chosen = logits.gather(1, ids)
    if over == G.GOLDY_ROUTER_ALL:
        w = torch.softmax(logits, 1).gather(1, ids)
    else:
        w = torch.softmax(chosen, 1)
    f = torch.zeros_like(x)
    for e in range(block.experts):
        t, j = (ids == e).nonzero(as_tuple=True)
        if len(t):
            o = ACT64[act](n[t] @ p["w1"][e] + p["b1"][e]) @ p["w2"][e] + p["b2"][e]
            f = f.index_add(0, t, w[t, j, None] * o)
    v = f
    if post != G.GOLDY_NORM_NONE:
        c = f - f.mean(1, keepdim=True) if post == G.GOLDY_NORM_LAYER else f
        v = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * p["gamma_f"] + p.get("beta_f", 0.0)
    y = alpha * x + p["gate"] * v
    y.backward(dy.double())
    return y.detach(), x.grad, {k: v.grad if v.grad is not None else torch.zeros_like(v) for k, v in p.items()}, logits.detach()


def near(got, ref, what, bound):
    assert torch.isfinite(got).all(), what
    off = float((got.double() - ref).norm() / ref.norm())
    assert off < bound, f"{what}: {off:.2e}"


@pytest.mark.parametrize("rows,width,hidden,experts,slots,act,post,alpha,over",
                         [(100, 136, 264, 8, 2, G.GOLDY_ACT_GELU, G.GOLDY_NORM_RMS, 1.0, G.GOLDY_ROUTER_ALL),
                          (513, 512, 1024, 16, 4, G.GOLDY_ACT_SILU, G.GOLDY_NORM_LAYER, 0.5, G.GOLDY_ROUTER_CHOSEN),
                          (300, 128, 512, 5, 5, G.GOLDY_ACT_GELU, G.GOLDY_NORM_NONE, 1.5, G.GOLDY_ROUTER_ALL),
                          (1, 256, 256, 64, 6, G.GOLDY_ACT_SILU, G.GOLDY_NORM_RMS, 1.0, G.GOLDY_ROUTER_CHOSEN),
                          (2000, 64, 128, 40, 3, G.GOLDY_ACT_NONE, G.GOLDY_NORM_RMS, 1.0, G.GOLDY_ROUTER_ALL)])
@pytest.mark.parametrize("keep8", [False, True])
def test_block(cuda_ok, rows, width, hidden, experts, slots, act, post, alpha, over, keep8):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows)
    block = RoutedFeedForward(rows, width, hidden, experts, slots, act, seed=1, post=post, alpha=alpha, keep8=keep8, over=over)
    x = torch.randn(rows, width, generator=gen, device="cuda").bfloat16()
    dy = torch.randn(rows, width, generator=gen, device="cuda").bfloat16()
    for k in ("b1", "b2", "beta_f"):
        if k in block.p:
            block.p[k].normal_(generator=gen).mul_(0.5)
    for k in ("gate", "gamma_f"):
        if k in block.p:
            block.p[k].add_(0.2 * torch.randn(width, generator=gen, device="cuda"))
    y = block.forward(x)
    dx = block.backward(dy)
    torch.cuda.synchronize()
    assert G.goldy_device_error(clear=True) == 0
    ry, rdx, rg, logits = reference(block, x, dy, act, post, alpha, over)
    # the choice: no logit left out is larger than a chosen one by more than both are off
    mine = torch.zeros_like(logits, dtype=torch.bool).scatter_(1, block.ids.long(), True)
    if slots < experts:
        out, least = logits.masked_fill(mine, -math.inf).amax(1), logits.masked_fill(~mine, math.inf).amin(1)
        assert (out - least <= 2e-2 * logits.abs().amax(1)).all()
    near(y, ry, "y", 2e-2)
    more = 8e-2 if keep8 else 0.0
    near(dx, rdx, "dx", 2e-2 + more)
    for k, ref in rg.items():
        if rows == 1 and k == "wr" or float(ref.norm()) < 1e-9:
            continue                                        # one row: a difference of few terms
        near(block.grads[k], ref, k, (3e-2 if k == "wr" else 2e-2) + more)


def test_kept_bytes(cuda_ok):
    """What stays of the hidden layer: 33 bytes per 32 pre-activations."""
    block = RoutedFeedForward(256, 64, 512, 4, 2, keep8=True)
    block.forward(torch.randn(256, 64, device="cuda").bfloat16())
    assert sum(t.numel() for t in block.q) == 512 * 512 * 33 // 32 and block.z is None and block.h is None


def test_replay(cuda_ok):
    """Both passes recorded in a CUDA graph give the bits of the eager calls."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    rnd = lambda: torch.randn(700, 128, generator=gen, device="cuda").bfloat16()  # noqa: E731
    for keep8 in (False, True):
        block = RoutedFeedForward(700, 128, 256, 12, 3, seed=2, keep8=keep8)
        x, dy = rnd(), rnd()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            block.forward(x)
            block.backward(dy)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = block.forward(x)
            dx = block.backward(dy)
        for _ in range(3):
            x.copy_(rnd())
            dy.copy_(rnd())
            graph.replay()
            torch.cuda.synchronize()
            got = [y.clone(), dx.clone()] + [block.grads[k].clone() for k in sorted(block.grads)]
            want = [block.forward(x), block.backward(dy)] + [block.grads[k] for k in sorted(block.grads)]
            for a, b in zip(got, want):
                assert torch.equal(a, b)
    assert G.goldy_device_error(clear=True) == 0


def test_command(cuda_ok, monkeypatch, capsys):
    """The command runs with a router and with pre-activations in 8 bits."""
    from paper_2409_02227_gb300 import ffn_block
    for more in ([], ["--keep8"]):
        monkeypatch.setattr("sys.argv", ["ffn_block", "--rows", "64", "--width", "64", "--hidden", "128", "--experts", "8", "--slots",
                                         "2", "--steps", "2"] + more)
        ffn_block.main()
        assert capsys.readouterr().out.count("loss") == 2
