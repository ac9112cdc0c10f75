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

``RoutedFeedForward`` chooses several experts per token by a router and joins
their weighted sum to the residual stream through a norm and a gate.

``python -m paper_2409_02227_gb300.ffn_block [--experts 8 [--slots 2 [--keep8]]]``
trains one block on a fixed synthetic batch for a few steps and prints the loss.
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


class RoutedFeedForward(FeedForward):
    """A block whose tokens go to several experts each, chosen by a router:

        n = norm(x),  logits = n Wr,  k experts e_j and weights w_j per token
        f = sum over j of w_j (act(n W1[e_j] + b1[e_j]) W2[e_j] + b2[e_j])
        y = alpha x + gate * post(f)

    ``post``: the norm after the block (a goldy_norm_kind); gate: one value per
    feature.  The products run on rows sorted by expert.  With ``keep8`` the
    pre-activations stay in 8 bits between the passes, and the hidden rows are made
    from them again; otherwise both stay in bf16."""

    def __init__(self, rows: int, width: int, hidden: int, experts: int, slots: int = 2, act: int = G.GOLDY_ACT_GELU,
                 seed: int = 0, device: str = "cuda", post: int = G.GOLDY_NORM_RMS, alpha: float = 1.0, keep8: bool = False,
                 over: int = G.GOLDY_ROUTER_ALL):
        if experts < 1 or not 1 <= slots <= min(experts, G.GOLDY_MAX_SLOTS):
            raise ValueError("a routed block needs experts, and 1 to as many slots per token")
        super().__init__(rows, width, hidden, experts, act, seed, device)
        gen = torch.Generator(device=device)
        gen.manual_seed(seed + 1)
        more = {"wr": (torch.randn(width, experts, generator=gen, device=device) * width ** -0.5).bfloat16(),
                "gate": torch.ones(width, device=device)}
        if post != G.GOLDY_NORM_NONE:
            more["gamma_f"] = torch.ones(width, device=device)
        if post == G.GOLDY_NORM_LAYER:
            more["beta_f"] = torch.zeros(width, device=device)
        self.p.update(more)
        self.grads.update({k: torch.empty(v.shape, device=device, dtype=torch.float32) for k, v in more.items()})
        self.slots, self.keep8 = slots, keep8
        self.z = self.h = None                                           # kept from pass to pass, of the experts' rows
        self.up = G.linear_desc(rows * slots, width, hidden, groups=experts, act=act, bias_dtype=G.GOLDY_F32)
        self.down = G.linear_desc(rows * slots, hidden, width, groups=experts, act_x=act, bias_dtype=G.GOLDY_F32)
        self.scores = G.linear_desc(rows, width, experts, y_dtype=G.GOLDY_F32, ldw=experts, ldy=experts)
        self.router = G.router_desc(rows, experts, slots, over=over)
        self.route = G.route_desc(rows, slots, experts, width)
        self.join = G.residual_norm_desc(rows, width, norm_f=post, norm_y=G.GOLDY_NORM_NONE, alpha=alpha)
        self.kept = G.keep8_desc(rows * slots, hidden, act=act)
        need = max([G.goldy_linear_query(d) for d in (self.up, self.down, self.scores)] +
                   [G.goldy_layernorm_query(self.norm), G.goldy_route_query(self.route), G.goldy_residual_norm_query(self.join)])
        self.work = torch.zeros(max(need, 256), dtype=torch.uint8, device=device)
        self.offsets = torch.empty(experts + 1, dtype=torch.int32, device=device)
        self.ids, self.place = (torch.empty(rows, slots, dtype=torch.int32, device=device) for _ in range(2))
        self.weights = torch.empty(rows, slots, device=device)
        self.logits = torch.empty(rows, experts, device=device)
        self.stats = torch.empty(4, rows, device=device)
        self.joined = self._params(self.p)

    def _params(self, t: Dict[str, torch.Tensor]) -> G.goldy_residual_norm_params:
        return G.residual_norm_params(**{k: t[k].data_ptr() for k in ("gate", "gamma_f", "beta_f") if k in t})

    def _rows(self, width: int) -> torch.Tensor:
        return torch.empty(self.rows * self.slots, width, device=self.work.device, dtype=torch.bfloat16)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """x: rows x width, bf16, any strides."""
        x = self.x = self._check(x, "x")
        p, kw = self.p, self._kw()
        dense, stream = dict(kw, offsets=0), kw["stream"]
        G.goldy_layernorm_forward(self.norm, x.data_ptr(), p["gamma"].data_ptr(), p["beta"].data_ptr(),
                                  self.normed.data_ptr(), self.mean.data_ptr(), self.rstd.data_ptr(), stream)
        G.goldy_linear_forward(self.scores, self.normed.data_ptr(), p["wr"].data_ptr(), self.logits.data_ptr(), **dense)
        G.goldy_router_forward(self.router, self.logits.data_ptr(), self.ids.data_ptr(), self.weights.data_ptr(), stream)
        G.goldy_route_sort(self.route, self.ids.data_ptr(), self.offsets.data_ptr(), self.place.data_ptr(), 0,
                           kw["workspace"], kw["workspace_bytes"], stream)
        self.e, self.out, z, h = (self._rows(w) for w in (self.width, self.width, self.kept.n, self.kept.n))
        G.goldy_route_dispatch(self.route, self.normed.data_ptr(), self.place.data_ptr(), self.e.data_ptr(), stream)
        G.goldy_linear_forward(self.up, self.e.data_ptr(), p["w1"].data_ptr(), h.data_ptr(), bias=p["b1"].data_ptr(),
                               z=z.data_ptr(), **kw)
        G.goldy_linear_forward(self.down, h.data_ptr(), p["w2"].data_ptr(), self.out.data_ptr(), bias=p["b2"].data_ptr(), **kw)
        self.f, y = torch.empty_like(x), torch.empty_like(x)
        G.goldy_route_combine(self.route, self.out.data_ptr(), self.place.data_ptr(), self.f.data_ptr(),
                              self.weights.data_ptr(), stream=stream)
        G.goldy_residual_norm_forward(self.join, self.joined, x.data_ptr(), self.f.data_ptr(), y.data_ptr(), 0,
                                      self.stats.data_ptr(), stream)
        if self.keep8:
            sizes = G.goldy_keep8_query(self.kept)
            self.q = tuple(torch.empty(max(b, 16), dtype=torch.uint8, device=x.device) for b in sizes)
            G.goldy_keep8_pack(self.kept, z.data_ptr(), self.q[0].data_ptr(), self.q[1].data_ptr(), stream)
        else:
            self.z, self.h = z, h
        return y

    def backward(self, dy: torch.Tensor) -> torch.Tensor:
        """The gradient of x; those of the parameters are in ``grads``."""
        if self.x is None:
            raise RuntimeError("backward needs a forward pass before it")
        dy = self._check(dy, "dy")
        p, g, kw = self.p, self.grads, self._kw()
        dense, stream, work = dict(kw, offsets=0), kw["stream"], (kw["workspace"], kw["workspace_bytes"])
        z, h = self.z, self.h
        if self.keep8:
            z, h = self._rows(self.kept.n), self._rows(self.kept.n)
            G.goldy_keep8_unpack(self.kept, self.q[0].data_ptr(), self.q[1].data_ptr(), z.data_ptr(), h.data_ptr(), stream)
        dx, df, dn, dstream = (torch.empty_like(dy) for _ in range(4))
        G.goldy_residual_norm_backward(self.join, self.joined, 0, dy.data_ptr(), self.f.data_ptr(), 0, self.stats.data_ptr(),
                                       dstream.data_ptr(), df.data_ptr(), self._params(g), *work, stream)
        dout, dz, de, dw = self._rows(self.width), torch.empty_like(z), torch.empty_like(self.e), torch.empty_like(self.weights)
        G.goldy_route_combine_grad(self.route, df.data_ptr(), self.out.data_ptr(), self.place.data_ptr(),
                                   self.weights.data_ptr(), dout.data_ptr(), dw.data_ptr(), stream)
        # the experts: down projection, whose input gradient is the up projection's dZ, and up projection
        G.goldy_linear_bias_grad(self.down, dout.data_ptr(), g["b2"].data_ptr(), **kw)
        G.goldy_linear_weight_grad(self.down, h.data_ptr(), dout.data_ptr(), g["w2"].data_ptr(), **kw)
        through = z.data_ptr() if self.down.act_x != G.GOLDY_ACT_NONE else 0
        G.goldy_linear_input_grad(self.down, dout.data_ptr(), p["w2"].data_ptr(), dz.data_ptr(), z=through, **kw)
        G.goldy_linear_bias_grad(self.up, dz.data_ptr(), g["b1"].data_ptr(), **kw)
        G.goldy_linear_weight_grad(self.up, self.e.data_ptr(), dz.data_ptr(), g["w1"].data_ptr(), **kw)
        G.goldy_linear_input_grad(self.up, dz.data_ptr(), p["w1"].data_ptr(), de.data_ptr(), **kw)
        # the normed rows: from their places, and through the router
        G.goldy_route_combine(self.route, de.data_ptr(), self.place.data_ptr(), dn.data_ptr(), stream=stream)
        dlogits = torch.empty_like(self.logits)
        G.goldy_router_backward(self.router, self.logits.data_ptr(), self.ids.data_ptr(), dw.data_ptr(), dlogits.data_ptr(), stream)
        # the products take bf16 rows: a rounding of the gradient that reaches wr and the normed rows
        dlogits = dlogits.bfloat16()
        G.goldy_linear_weight_grad(self.scores, self.normed.data_ptr(), dlogits.data_ptr(), g["wr"].data_ptr(), **dense)
        G.goldy_linear_input_grad(self.scores, dlogits.data_ptr(), p["wr"].data_ptr(), dn.data_ptr(), residual=dn.data_ptr(), **dense)
        G.goldy_layernorm_backward(self.norm, dn.data_ptr(), self.x.data_ptr(), p["gamma"].data_ptr(), self.mean.data_ptr(),
                                   self.rstd.data_ptr(), dx.data_ptr(), g["gamma"].data_ptr(), g["beta"].data_ptr(), *work, stream)
        G.goldy_ewise_add(dx.data_ptr(), dstream.data_ptr(), dx.data_ptr(), dx.numel(), G.GOLDY_BF16, 1, stream)
        return dx


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rows", type=int, default=2048)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--experts", type=int, default=0)
    ap.add_argument("--slots", type=int, default=0, help="experts per token, chosen by a router")
    ap.add_argument("--keep8", action="store_true", help="keep pre-activations in 8 bits (with --slots)")
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--rate", type=float, default=1e-4)
    a = ap.parse_args()
    if a.keep8 and not a.slots:
        ap.error("--keep8 goes with --slots")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.randn(a.rows, a.width, generator=gen, device="cuda").bfloat16()
    target = torch.randn(a.rows, a.width, generator=gen, device="cuda").bfloat16()
    inputs = [x]
    if a.slots:
        block = RoutedFeedForward(a.rows, a.width, a.hidden, a.experts, a.slots, keep8=a.keep8)
    else:
        inputs.append(torch.randint(0, a.experts, (a.rows,), generator=gen, device="cuda") if a.experts else None)
        block = FeedForward(a.rows, a.width, a.hidden, a.experts)
    for step in range(a.steps):
        y = block.forward(*inputs)
        error = y.float() - target.float()
        print(f"step {step}: loss {float(error.square().sum(1).mean()):.3f}")
        block.backward((error * (2.0 / a.rows)).bfloat16())
        block.step(a.rate)
    if G.goldy_device_error(clear=True) != 0:
        raise RuntimeError("a kernel gave up a bounded wait")


if __name__ == "__main__":
    main()
