"""A Transformer feed-forward block on the layer operators, forwards and
backwards, dense or with experts:

    y = x + act(norm(x) W1 + b1) W2 + b2

Every step is one call of the library: layer norm, the two products with bias,
activation and residual in their epilogues, and in the backward pass the
input gradient through the activation, weight gradients, bias gradients and
the norm's gradient.  With experts, token r goes through the weights of expert
ids[r]: rows are ordered by expert once, and the products take the experts'
row ranges from an offsets array on the device.  A token whose id is no
expert's goes through none: its y is x, and it adds to no gradient but dx.

``python -m paper_2409_02227_gb300.ffn_block [--experts 8]`` trains one block
on a fixed synthetic batch for a few steps and prints the loss.
"""
from __future__ import annotations

import argparse
from typing import Dict, Optional

import torch

from . import goldy as G


class FeedForward:
    """Weights in bf16, norm parameters and biases in fp32; gradients of all
    of them in fp32, in ``grads`` after ``backward``."""

    def __init__(self, rows: int, width: int, hidden: int, experts: int = 0, act: int = G.GOLDY_ACT_GELU,
                 seed: int = 0, device: str = "cuda"):
        if width % 8 or hidden % 8:
            raise ValueError("width and hidden must be multiples of 8")
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        lead = (experts,) if experts else ()
        rnd = lambda *s: torch.randn(*s, generator=gen, device=device)  # noqa: E731
        self.experts, self.rows, self.width = experts, rows, width
        self.p: Dict[str, torch.Tensor] = {
            "gamma": torch.ones(width, device=device), "beta": torch.zeros(width, device=device),
            "w1": (rnd(*lead, width, hidden) * width ** -0.5).bfloat16(), "b1": torch.zeros(*lead, hidden, device=device),
            "w2": (rnd(*lead, hidden, width) * hidden ** -0.5).bfloat16(), "b2": torch.zeros(*lead, width, device=device)}
        self.grads = {k: torch.empty(v.shape, device=device, dtype=torch.float32) for k, v in self.p.items()}
        row = lambda n, dtype=torch.bfloat16: torch.empty(rows, n, device=device, dtype=dtype)  # noqa: E731
        self.normed, self.z, self.h = row(width), row(hidden), row(hidden)
        self.mean, self.rstd = (torch.empty(rows, device=device) for _ in range(2))
        # the second layer's input gradient goes through the first one's activation
        self.norm = G.layernorm_desc(rows, width, param_dtype=G.GOLDY_F32)
        self.up = G.linear_desc(rows, width, hidden, groups=experts, act=act, bias_dtype=G.GOLDY_F32)
        self.down = G.linear_desc(rows, hidden, width, groups=experts, act_x=act, bias_dtype=G.GOLDY_F32)
        need = max(G.goldy_linear_query(self.up), G.goldy_linear_query(self.down), G.goldy_layernorm_query(self.norm))
        self.work = torch.zeros(max(need, 256), dtype=torch.uint8, device=device)
        self.master: Optional[Dict[str, torch.Tensor]] = None
        self.x: Optional[torch.Tensor] = None            # the forward pass's rows
        self.order: Optional[torch.Tensor] = None
        self.offsets: Optional[torch.Tensor] = None
        self.lost: Optional[torch.Tensor] = None         # rows without an expert, in the experts' order
        self.bounds = torch.arange(experts + 1, device=device)
        self.zero = torch.zeros((), device=device, dtype=torch.bfloat16)

    def _kw(self):
        if not self.work.is_cuda:
            raise RuntimeError(f"the block is on {self.work.device}: its kernels need a GPU")
        return dict(offsets=0 if self.offsets is None else self.offsets.data_ptr(), workspace=self.work.data_ptr(),
                    workspace_bytes=self.work.numel(), stream=torch.cuda.current_stream().cuda_stream)

    def _check(self, t: torch.Tensor, name: str) -> torch.Tensor:
        """A tensor for the kernels, which take an address: rows packed and on a
        16-byte boundary, copied if they are not."""
        shape = (self.rows, self.width)
        if t.shape != shape or t.dtype != torch.bfloat16 or t.device != self.work.device:
            raise ValueError(f"{name} must be a bf16 tensor of {shape[0]} x {shape[1]} on {self.work.device}, "
                             f"not {t.dtype} of {' x '.join(map(str, t.shape))} on {t.device}")
        t = t.contiguous()
        return t.clone() if t.data_ptr() % 16 else t

    def _route(self, ids: Optional[torch.Tensor]) -> None:
        if (ids is not None) != (self.experts > 0):
            raise ValueError("expert ids come with experts")
        if ids is None:
            return
        whole = ids.dtype in (torch.uint8, torch.int8, torch.int16, torch.int32, torch.int64)
        if ids.shape != (self.rows,) or not whole or ids.device != self.work.device:
            raise ValueError(f"ids must be {self.rows} integers on {self.work.device}, "
                             f"not {ids.dtype} of {' x '.join(map(str, ids.shape))} on {ids.device}")
        ids, self.order = ids.long().sort(stable=True)
        self.offsets = torch.searchsorted(ids, self.bounds, out_int32=True)
        self.lost = (ids.clamp(0, self.experts - 1) != ids)[:, None]

    def forward(self, x: torch.Tensor, ids: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x: rows x width, bf16, any strides; ids: the expert of each row."""
        x = self._check(x, "x")
        self._route(ids)
        p, kw = self.p, self._kw()
        if ids is None:
            self.x, y = x, torch.empty_like(x)
        else:
            # rows without an expert: y keeps x, which the products leave as it is,
            # and the norm sees zeros
            y = x[self.order]
            self.x = torch.where(self.lost, self.zero, y)
        G.goldy_layernorm_forward(self.norm, self.x.data_ptr(), p["gamma"].data_ptr(), p["beta"].data_ptr(),
                                  self.normed.data_ptr(), self.mean.data_ptr(), self.rstd.data_ptr(), kw["stream"])
        G.goldy_linear_forward(self.up, self.normed.data_ptr(), p["w1"].data_ptr(), self.h.data_ptr(),
                               bias=p["b1"].data_ptr(), z=self.z.data_ptr(), **kw)
        G.goldy_linear_forward(self.down, self.h.data_ptr(), p["w2"].data_ptr(), y.data_ptr(), bias=p["b2"].data_ptr(),
                               residual=self.x.data_ptr(), **kw)
        return y if ids is None else torch.empty_like(y).index_copy_(0, self.order, y)

    def backward(self, dy: torch.Tensor) -> torch.Tensor:
        """The gradient of x; those of the parameters are in ``grads``."""
        if self.x is None:
            raise RuntimeError("backward needs a forward pass before it")
        dy = self._check(dy, "dy")
        p, g, kw = self.p, self.grads, self._kw()
        dy = dy if self.order is None else dy[self.order]
        dz, dx = torch.empty_like(self.z), torch.empty_like(self.x)
        dnormed = torch.empty_like(self.normed) if self.order is None else torch.zeros_like(self.normed)
        # down projection; its input gradient is the up projection's dZ
        G.goldy_linear_bias_grad(self.down, dy.data_ptr(), g["b2"].data_ptr(), **kw)
        G.goldy_linear_weight_grad(self.down, self.h.data_ptr(), dy.data_ptr(), g["w2"].data_ptr(), **kw)
        z = self.z.data_ptr() if self.down.act_x != G.GOLDY_ACT_NONE else 0
        G.goldy_linear_input_grad(self.down, dy.data_ptr(), p["w2"].data_ptr(), dz.data_ptr(), z=z, **kw)
        # up projection
        G.goldy_linear_bias_grad(self.up, dz.data_ptr(), g["b1"].data_ptr(), **kw)
        G.goldy_linear_weight_grad(self.up, self.normed.data_ptr(), dz.data_ptr(), g["w1"].data_ptr(), **kw)
        G.goldy_linear_input_grad(self.up, dz.data_ptr(), p["w1"].data_ptr(), dnormed.data_ptr(), **kw)
        # norm, and the residual's share
        G.goldy_layernorm_backward(self.norm, dnormed.data_ptr(), self.x.data_ptr(), p["gamma"].data_ptr(),
                                   self.mean.data_ptr(), self.rstd.data_ptr(), dx.data_ptr(), g["gamma"].data_ptr(),
                                   g["beta"].data_ptr(), self.work.data_ptr(), self.work.numel(), kw["stream"])
        G.goldy_ewise_add(dx.data_ptr(), dy.data_ptr(), dx.data_ptr(), dx.numel(), G.GOLDY_BF16, 1, kw["stream"])
        return dx if self.order is None else torch.empty_like(dx).index_copy_(0, self.order, dx)

    def step(self, rate: float) -> None:
        """Plain gradient descent, on fp32 copies of the parameters."""
        if self.master is None:
            self.master = {k: v.float() for k, v in self.p.items()}
        for k, v in self.master.items():
            v -= rate * self.grads[k]
            self.p[k].copy_(v)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rows", type=int, default=2048)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--experts", type=int, default=0)
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--rate", type=float, default=1e-4)
    a = ap.parse_args()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.randn(a.rows, a.width, generator=gen, device="cuda").bfloat16()
    target = torch.randn(a.rows, a.width, generator=gen, device="cuda").bfloat16()
    ids = torch.randint(0, a.experts, (a.rows,), generator=gen, device="cuda") if a.experts else None
    block = FeedForward(a.rows, a.width, a.hidden, a.experts)
    for step in range(a.steps):
        y = block.forward(x, ids)
        error = y.float() - target.float()
        print(f"step {step}: loss {float(error.square().sum(1).mean()):.3f}")
        block.backward((error * (2.0 / a.rows)).bfloat16())
        block.step(a.rate)
    if G.goldy_device_error(clear=True) != 0:
        raise RuntimeError("a kernel gave up a bounded wait")


if __name__ == "__main__":
    main()
