"""Measured cases of the operators around a feed-forward block with experts:
the router (k experts and weights per token, and the logits' gradient), tokens
sorted by expert and back with the weights applied, and their gradient, the
norms before and after a block fused with its gate and residual scale, forwards
and backwards, and pre-activations kept in 8 bits for the backward pass.

Every case runs through ``run`` in one of two forms: elementary torch
operations in fp32 (``own`` false) or the calls a user makes of the package
(``own`` true).  ``exact`` gives the same results from the definitions in fp64.

A case is a dict of plain values:

  op        "router" (forward), "router_step" (forward and backward),
            "dispatch" (tokens sorted by expert, their rows copied there),
            "combine" (rows of a token's experts, weighted, summed),
            "combine_grad", "norms", "norms_grad", or
            "keep" (8 bits written, then read back as Z and act(Z))
  rows      tokens
  experts, k   experts, and slots per token
  over      router: softmax over "all" experts or over the "chosen" ones
  width, n  features of a row
  dtype     type of rows or logits ("bf16" or "f32")
  weighted, residual   combine: which of them are there
  norm_f, norm_y, gate, alpha   norms: S = alpha X + gate * N_f(F), Y = N_y(S);
            kinds "none", "layer" or "rms"
  act       keep: the activation of the rows that are read back
"""
from __future__ import annotations

import math
import random

import torch

own = False

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
BLOCK = 32                   # kept elements that share a scale
MOST_LOGITS = 32768 * 128
MOST_VALUES = 3 * 16384 * 4096        # elements moved by a routing case
MOST_NORM = 16384 * 4096
MOST_KEPT = 8192 * 8192


def router(name, op, rows, experts, k, over="all", dtype="f32", scale=1.0):
    return {"name": name, "op": op, "rows": rows, "experts": experts, "k": k, "over": over, "dtype": dtype, "scale": scale}


def route(name, op, rows, experts, k, width, dtype="bf16", weighted=True, residual=False):
    return {"name": name, "op": op, "rows": rows, "experts": experts, "k": k, "width": width, "dtype": dtype,
            "weighted": weighted, "residual": residual}


def norms(name, op, rows, n, dtype="bf16", norm_f="rms", norm_y="rms", gate=True, alpha=1.0):
    return {"name": name, "op": op, "rows": rows, "n": n, "dtype": dtype, "norm_f": norm_f, "norm_y": norm_y,
            "gate": gate, "alpha": alpha}


def keep(name, rows, n, act="gelu", dtype="bf16"):
    return {"name": name, "op": "keep", "rows": rows, "n": n, "act": act, "dtype": dtype}


def listed():
    return [
        # a decoding batch picks its experts: latency counts
        router("router_decode", "router", 16, 64, 6, over="chosen"),
        # a training batch, forwards and backwards
        router("router_train", "router_step", 32768, 128, 8),
        # the decoding batch's rows go to their experts: two short launches
        route("dispatch_decode", "dispatch", 16, 64, 6, 2048),
        # a training batch over few experts
        route("dispatch_train", "dispatch", 16384, 16, 2, 4096),
        # the experts' rows come back, many slots per token, residual added
        route("combine_train", "combine", 8192, 64, 8, 2048, residual=True),
        # the way back: rows' gradients to the experts, and the weights' gradient;
        # odd sizes, rows off a vector's boundary
        route("combine_grad_odd", "combine_grad", 5000, 31, 3, 1111),
        # one token's residual: latency only
        norms("norms_token", "norms", 1, 4096, norm_f="layer", norm_y="layer"),
        # a training batch
        norms("norms_train", "norms", 16384, 4096),
        norms("norms_grad", "norms_grad", 16384, 2048, alpha=0.5),
        # fp32 with an odd row length
        norms("norms_grad_odd_f32", "norms_grad", 1000, 1023, dtype="f32", norm_f="layer", norm_y="layer"),
        # a small batch's pre-activations, rows that end inside a block
        keep("keep_small", 100, 1000, act="silu"),
        # a training batch's
        keep("keep_train", 8192, 8192),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A feature count: half of the time a multiple of 64, else any."""
    v = _log(rng, lo, hi)
    return max(lo, 64 * round(v / 64)) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["router", "router_step", "dispatch", "combine", "combine_grad", "norms", "norms", "norms_grad",
                     "norms_grad", "keep"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("norms", "norms_grad"):
        while True:
            rows, n = _log(rng, 1, 16384), _size(rng, 16, 8192)
            if rows * n * (1 if dtype == "bf16" else 2) <= MOST_NORM // (2 if op == "norms_grad" else 1):
                break
        return {"op": op, "rows": rows, "n": n, "dtype": dtype, "norm_f": rng.choice(["none", "layer", "rms", "rms"]),
                "norm_y": rng.choice(["layer", "rms", "rms"]), "gate": rng.random() < 0.7,
                "alpha": rng.choice([1.0, 1.0, 0.5, round(rng.uniform(0.1, 2.0), 3)])}
    if op == "keep":
        while True:
            rows, n = _log(rng, 1, 32768), _size(rng, 16, 16384)
            if rows * n * (1 if dtype == "bf16" else 2) <= MOST_KEPT:
                return {"op": op, "rows": rows, "n": n, "dtype": dtype, "act": rng.choice(ACTS)}
    experts = rng.choice([4, 8, 16, 31, 60, 64, 128, 256])
    k = rng.randint(1, min(8, experts))
    if op in ("router", "router_step"):
        while True:
            rows = _log(rng, 1, 32768)
            if rows * experts <= MOST_LOGITS:
                return {"op": op, "rows": rows, "experts": experts, "k": k, "over": rng.choice(["all", "chosen"]),
                        "dtype": dtype, "scale": rng.choice([1.0, 2.5])}
    while True:
        rows, width = _log(rng, 1, 32768), _size(rng, 64, 8192)
        values = rows * width * (2 * k + 1 if op == "combine_grad" else k + 2) * (1 if dtype == "bf16" else 2)
        if values <= MOST_VALUES:
            return {"op": op, "rows": rows, "experts": experts, "k": k, "width": width, "dtype": dtype,
                    "weighted": rng.random() < 0.7, "residual": rng.random() < 0.5}


# ---- inputs -------------------------------------------------------------------

def _logits(case, gen):
    """A router's outputs: experts of uneven popularity; one in sixteen closed
    to every token, padding rows open to none."""
    rows, experts = case["rows"], case["experts"]
    popular = torch.randn(experts, generator=gen, device="cuda")
    l = 1.5 * torch.randn(rows, experts, generator=gen, device="cuda") + 0.7 * popular
    l = l.to(TYPES[case["dtype"]])
    if experts >= 16:
        l[:, torch.randperm(experts, generator=gen, device="cuda")[:experts // 16]] = -math.inf
    if rows >= 64:
        l[rows - rows // 64:] = -math.inf
    return l


def _ids(case, gen):
    """k different experts per token, popular ones more often; one slot in
    thirty is dropped (an expert that was full)."""
    rows, experts = case["rows"], case["experts"]
    score = torch.rand(rows, experts, generator=gen, device="cuda").log_().neg_().log_().neg_()
    score += 0.7 * torch.randn(experts, generator=gen, device="cuda")
    ids = torch.topk(score, case["k"], dim=1).indices.int()
    ids[torch.rand(ids.shape, generator=gen, device="cuda") < 1 / 30] = -1
    return ids


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    rnd = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    rows, op, dtype = case["rows"], case["op"], TYPES[case["dtype"]]
    if op in ("router", "router_step"):
        s["logits"] = _logits(case, gen)
        if op == "router_step":
            s["dweights"] = 0.01 * rnd(rows, case["k"])
    elif op in ("norms", "norms_grad"):
        _prepare_norms(s, case, rnd, gen)
    elif op == "keep":
        # pre-activations: features of different sizes, a few rows large
        n = case["n"]
        z = rnd(rows, n) * torch.exp(0.5 * rnd(n)) * (1.0 + 9.0 * (torch.rand(rows, 1, generator=gen, device="cuda") < 0.02))
        s["z"] = z.to(dtype)
    else:
        k, width = case["k"], case["width"]
        s["ids"] = _ids(case, gen)
        if op == "dispatch":
            s["x"] = rnd(rows, width).to(dtype)
        else:
            sorted_ = _sort(s["ids"], case["experts"])
            s["place"] = sorted_["place"]
            s["e"] = rnd(rows * k, width).to(dtype)
            s["weights"] = torch.softmax(rnd(rows, k), 1)
            if op == "combine_grad":
                s["dy"] = (0.01 * rnd(rows, width)).to(dtype)
            else:
                if not case["weighted"]:
                    s["weights"] = None
                s["r"] = rnd(rows, width).to(dtype) if case["residual"] else None
    if own:
        _plan(s)
    return s


def _prepare_norms(s, case, rnd, gen):
    rows, n, dtype = case["rows"], case["n"], TYPES[case["dtype"]]
    # a residual stream: a few features stand out, and the mean is not 0
    feature, scale = rnd(n), 1.0 + 4.0 * (torch.rand(n, generator=gen, device="cuda") < 0.02)
    stream = (rnd(rows, n) * scale + 0.3 * feature + 0.1).to(dtype)
    s["f"] = (0.5 * rnd(rows, n) + 0.2 * rnd(n)).to(dtype)
    for name, kind in (("f", case["norm_f"]), ("y", case["norm_y"])):
        s["gamma_" + name] = 1.0 + 0.1 * rnd(n) if kind != "none" else None
        s["beta_" + name] = 0.1 * rnd(n) if kind == "layer" else None
    s["gate"] = 0.3 + 0.1 * rnd(n) if case["gate"] else None
    if case["op"] == "norms":
        s["x"] = stream
        return
    s["s"] = stream
    s["dy"], s["ds"] = ((0.01 * rnd(rows, n)).to(dtype) for _ in range(2))
    s["stats"] = torch.zeros(4, rows, device="cuda")
    for i, (t, kind) in enumerate(((s["f"], case["norm_f"]), (stream, case["norm_y"]))):
        if kind == "none":
            continue
        v = t.double()
        if kind == "layer":
            s["stats"][2 * i] = v.mean(1)
            v = v - v.mean(1, keepdim=True)
        s["stats"][2 * i + 1] = torch.rsqrt((v * v).mean(1) + EPS)


# ---- the calls a user makes -----------------------------------------------------

def _plan(s):
    """What a user's program keeps: descriptors, output buffers, a workspace."""
    from paper_2409_02227_gb300 import goldy as G

    case, rows, op = s["case"], s["case"]["rows"], s["case"]["op"]
    s["G"], dtype = G, {"bf16": G.GOLDY_BF16, "f32": G.GOLDY_F32}[case["dtype"]]
    empty = lambda *shape, dtype=TYPES[case["dtype"]]: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    whole = lambda *shape: empty(*shape, dtype=torch.int32)  # noqa: E731
    f32 = lambda *shape: empty(*shape, dtype=torch.float32)  # noqa: E731
    need = 0
    if op in ("router", "router_step"):
        over = G.GOLDY_ROUTER_ALL if case["over"] == "all" else G.GOLDY_ROUTER_CHOSEN
        s["desc"] = G.router_desc(rows, case["experts"], case["k"], dtype=dtype, over=over, scale=case["scale"])
        s["chosen"], s["w"] = whole(rows, case["k"]), f32(rows, case["k"])
        if op == "router_step":
            s["dlogits"] = torch.empty_like(s["logits"])
    elif op in ("norms", "norms_grad"):
        kind = {"none": G.GOLDY_NORM_NONE, "layer": G.GOLDY_NORM_LAYER, "rms": G.GOLDY_NORM_RMS}
        n, names = case["n"], ("gate", "gamma_f", "beta_f", "gamma_y", "beta_y")
        s["desc"] = d = G.residual_norm_desc(rows, n, norm_f=kind[case["norm_f"]], norm_y=kind[case["norm_y"]], dtype=dtype,
                                             param_dtype=G.GOLDY_F32, eps=EPS, alpha=case["alpha"])
        s["params"] = G.residual_norm_params(**{p: _ptr(s, p) for p in names})
        if op == "norms":
            s["s"], s["y"], s["stats"] = torch.empty_like(s["x"]), torch.empty_like(s["x"]), f32(4, rows)
            s["out"] = dict(_stats(case, s["stats"]), s=s["s"], y=s["y"])
        else:
            s["dx"], s["df"] = torch.empty_like(s["s"]), torch.empty_like(s["s"])
            s["grads"] = {p: f32(n) for p in names if s[p] is not None}
            s["grad_ptrs"] = G.residual_norm_params(**{p: t.data_ptr() for p, t in s["grads"].items()})
            need = G.goldy_residual_norm_query(d)
    elif op == "keep":
        n = case["n"]
        s["desc"] = d = G.keep8_desc(rows, n, dtype=dtype, act=getattr(G, "GOLDY_ACT_" + case["act"].upper()))
        q_bytes, scale_bytes = G.goldy_keep8_query(d)
        s["q"], s["scales"] = (torch.empty(b, dtype=torch.uint8, device="cuda") for b in (q_bytes, scale_bytes))
        s["z8"], s["h"] = torch.empty_like(s["z"]), torch.empty_like(s["z"])
    else:
        k, width = case["k"], case["width"]
        s["desc"] = d = G.route_desc(rows, k, case["experts"], width, dtype=dtype)
        if op == "dispatch":
            s["offsets"], s["place"], s["source"] = whole(case["experts"] + 1), whole(rows, k), whole(rows * k)
            s["e"] = empty(rows * k, width).zero_()      # rows behind the last expert's stay as they are
            need = G.goldy_route_query(d)
        elif op == "combine":
            s["y"] = empty(rows, width)
        else:
            s["de"], s["dweights"] = empty(rows * k, width).zero_(), f32(rows, k)
    s["work"] = torch.zeros(max(need, 256), dtype=torch.uint8, device="cuda")


def _ptr(s, name):
    t = s.get(name)
    return 0 if t is None else t.data_ptr()


def _run_own(s):
    G, d, case, op = s["G"], s["desc"], s["case"], s["case"]["op"]
    stream = torch.cuda.current_stream().cuda_stream
    if op in ("router", "router_step"):
        G.goldy_router_forward(d, _ptr(s, "logits"), _ptr(s, "chosen"), _ptr(s, "w"), stream=stream)
        out = {"ids": s["chosen"], "weights": s["w"]}
        if op == "router_step":
            G.goldy_router_backward(d, _ptr(s, "logits"), _ptr(s, "chosen"), _ptr(s, "dweights"), _ptr(s, "dlogits"),
                                    stream=stream)
            out["dlogits"] = s["dlogits"]
        return out
    if op == "norms":
        G.goldy_residual_norm_forward(d, s["params"], _ptr(s, "x"), _ptr(s, "f"), _ptr(s, "s"), _ptr(s, "y"),
                                      stats=_ptr(s, "stats"), stream=stream)
        return s["out"]
    if op == "norms_grad":
        G.goldy_residual_norm_backward(d, s["params"], _ptr(s, "dy"), _ptr(s, "ds"), _ptr(s, "f"), _ptr(s, "s"),
                                       _ptr(s, "stats"), _ptr(s, "dx"), _ptr(s, "df"), s["grad_ptrs"],
                                       workspace=_ptr(s, "work"), workspace_bytes=s["work"].numel(), stream=stream)
        return dict({"d" + p: t for p, t in s["grads"].items()}, dx=s["dx"], df=s["df"])
    if op == "keep":
        G.goldy_keep8_pack(d, _ptr(s, "z"), _ptr(s, "q"), _ptr(s, "scales"), stream=stream)
        G.goldy_keep8_unpack(d, _ptr(s, "q"), _ptr(s, "scales"), _ptr(s, "z8"), _ptr(s, "h"), stream=stream)
        return {"z": s["z8"], "h": s["h"]}
    if op == "dispatch":
        G.goldy_route_sort(d, _ptr(s, "ids"), _ptr(s, "offsets"), _ptr(s, "place"), source=_ptr(s, "source"),
                           workspace=_ptr(s, "work"), workspace_bytes=s["work"].numel(), stream=stream)
        G.goldy_route_dispatch(d, _ptr(s, "x"), _ptr(s, "place"), _ptr(s, "e"), stream=stream)
        return {k: s[k] for k in ("offsets", "place", "source", "e")}
    if op == "combine":
        G.goldy_route_combine(d, _ptr(s, "e"), _ptr(s, "place"), _ptr(s, "y"), weights=_ptr(s, "weights"),
                              residual=_ptr(s, "r"), stream=stream)
        return {"y": s["y"]}
    G.goldy_route_combine_grad(d, _ptr(s, "dy"), _ptr(s, "e"), _ptr(s, "place"), _ptr(s, "weights"), _ptr(s, "de"),
                               _ptr(s, "dweights"), stream=stream)
    return {"de": s["de"], "dweights": s["dweights"]}


def _stats(case, stats):
    """The statistics that the norms of a case have."""
    out = {}
    for i, (name, kind) in enumerate((("f", case["norm_f"]), ("y", case["norm_y"]))):
        if kind == "layer":
            out["mean_" + name] = stats[2 * i]
        if kind != "none":
            out["rstd_" + name] = stats[2 * i + 1]
    return out


# ---- the plain form ---------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, 0.0, z)
    if act == "gelu":
        return z * (0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _choose(logits, k):
    """The k largest of each row, ties to the lowest index; -1 where only closed
    experts are left."""
    best, at = torch.sort(logits, dim=1, descending=True, stable=True)
    return torch.where(best[:, :k] == -math.inf, -1, at[:, :k]).int()


def _probabilities(case, l, ids):
    """Softmax over all experts, or over the chosen ones (0 elsewhere); 0 in rows
    without an open expert."""
    if case["over"] == "chosen":
        taken = torch.zeros_like(l, dtype=torch.bool)
        taken.scatter_(1, ids.clamp(min=0).long(), True)     # a row without a chosen expert is closed anyhow
        l = torch.where(taken, l, -math.inf)
    top = l.amax(1, keepdim=True)
    p = torch.exp(l - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(1, keepdim=True)
    return torch.where(total > 0, p / total, 0.0)


def _at(t, ids):
    return torch.where(ids < 0, 0.0, t.gather(1, ids.clamp(min=0).long()))


def _sort(ids, experts):
    """Slots by expert, in their order; slots without an expert behind them."""
    flat = ids.flatten()
    key = torch.where((flat < 0) | (flat >= experts), experts, flat)
    by, order = torch.sort(key, stable=True)
    offsets = torch.searchsorted(by, torch.arange(experts + 1, device=by.device, dtype=by.dtype), out_int32=True)
    place = torch.empty_like(order).scatter_(0, order, torch.arange(len(order), device=order.device))
    return {"offsets": offsets, "place": torch.where(key == experts, -1, place).int().view(ids.shape),
            "source": torch.where(by == experts, -1, order).int()}


def _quantised(z):
    """e4m3 multiples of a power of two per block of a row: the smallest power
    that keeps the block's largest value within 448."""
    rows, n = z.shape
    pad = torch.cat([z, z.new_zeros(rows, -n % BLOCK)], 1).view(rows, -1, BLOCK)
    m, e = torch.frexp(pad.abs().amax(2, keepdim=True))      # m in [1/2, 1)
    e = torch.where(m == 0, -127, torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-127)).int()
    power = lambda i: torch.where(i > -127, (i + 127) << 23, 1 << 22).int().view(torch.float32)  # noqa: E731
    v = pad * power(-e)
    step = torch.frexp(v)[1].sub(1).clamp(min=-6) - 3        # v's own power of two, or the smallest normal's
    q = torch.round(v * power(-step)) * power(step)
    return (q * power(e)).view(rows, -1)[:, :n]


def _norm(x, kind, gamma, beta):
    """The norm of x, its mean and 1 / deviation."""
    if kind == "none":
        return x, None, None
    mean = x.mean(1, keepdim=True) if kind == "layer" else None
    c = x - mean if kind == "layer" else x
    rstd = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
    y = c * rstd * gamma
    return (y if beta is None else y + beta), mean, rstd


def _run_plain(s):
    case, op = s["case"], s["case"]["op"]
    dtype = TYPES[case["dtype"]]
    if op in ("router", "router_step"):
        l, scale = s["logits"].float(), case["scale"]
        ids = _choose(l, case["k"])
        p = _probabilities(case, l, ids)
        out = {"ids": ids, "weights": scale * _at(p, ids)}
        if op == "router_step":
            g = torch.zeros_like(p)
            g.scatter_add_(1, ids.clamp(min=0).long(), torch.where(ids < 0, 0.0, scale * s["dweights"]))
            out["dlogits"] = (p * (g - (g * p).sum(1, keepdim=True))).to(dtype)
        return out
    if op == "norms":
        nf, mean_f, rstd_f = _norm(s["f"].float(), case["norm_f"], s["gamma_f"], s["beta_f"])
        t = case["alpha"] * s["x"].float() + (nf if s["gate"] is None else s["gate"] * nf)
        y, mean_y, rstd_y = _norm(t, case["norm_y"], s["gamma_y"], s["beta_y"])
        out = {"s": t.to(dtype), "y": y.to(dtype), "mean_f": mean_f, "rstd_f": rstd_f, "mean_y": mean_y, "rstd_y": rstd_y}
        return {k: v[:, 0] if k[:4] in ("mean", "rstd") else v for k, v in out.items() if v is not None}
    if op == "norms_grad":
        stats = s["stats"][:, :, None]
        grads = {}

        def back(g, x, kind, gamma, mean, rstd, name):
            if kind == "none":
                return g
            xhat = (x - mean) * rstd if kind == "layer" else x * rstd
            grads["dgamma_" + name] = (g * xhat).sum(0)
            if kind == "layer":
                grads["dbeta_" + name] = g.sum(0)
            g = g * gamma
            d = g - xhat * (g * xhat).mean(1, keepdim=True)
            return rstd * (d - g.mean(1, keepdim=True) if kind == "layer" else d)

        t = s["ds"].float() + back(s["dy"].float(), s["s"].float(), case["norm_y"], s["gamma_y"], stats[2], stats[3], "y")
        u, f = t, s["f"].float()
        if s["gate"] is not None:
            nf = f
            if case["norm_f"] != "none":
                nf = (f - stats[0]) * stats[1] * s["gamma_f"] if case["norm_f"] == "layer" else f * stats[1] * s["gamma_f"]
                nf = nf if s["beta_f"] is None else nf + s["beta_f"]
            grads["dgate"] = (t * nf).sum(0)
            u = t * s["gate"]
        df = back(u, f, case["norm_f"], s["gamma_f"], stats[0], stats[1], "f")
        return dict(grads, dx=(case["alpha"] * t).to(dtype), df=df.to(dtype))
    if op == "keep":
        z = _quantised(s["z"].float())
        return {"z": z.to(dtype), "h": _act(z, case["act"]).to(dtype)}
    if op == "dispatch":
        out = _sort(s["ids"], case["experts"])
        at = out["source"][:, None]
        return dict(out, e=torch.where(at < 0, 0.0, s["x"][at[:, 0].clamp(min=0).long() // case["k"]].float()).to(dtype))
    place = s["place"].long()
    if op == "combine":
        e = torch.where(place[:, :, None] < 0, 0.0, s["e"][place.clamp(min=0)].float())
        y = e.sum(1) if s["weights"] is None else (e * s["weights"][:, :, None]).sum(1)
        return {"y": (y if s["r"] is None else y + s["r"].float()).to(dtype)}
    lost = place < 0
    dy = s["dy"].float()
    dw = (torch.where(lost[:, :, None], 0.0, s["e"][place.clamp(min=0)].float()) * dy[:, None]).sum(2)
    de = torch.zeros(place.numel() + 1, dy.shape[1], device=dy.device)       # the last row takes what is lost
    de[torch.where(lost, place.numel(), place)] = dy[:, None] * s["weights"][:, :, None]
    return {"de": de[:-1].to(dtype), "dweights": dw}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ---------------------------------------------------

def work(case):
    """Each input read once and each output written once."""
    rows, op, size = case["rows"], case["op"], 2 if case["dtype"] == "bf16" else 4
    if op in ("router", "router_step"):
        step = op == "router_step"
        b = rows * case["experts"] * size * (2 if step else 1) + 8 * rows * case["k"] + 4 * rows * case["k"] * step
        return {"bytes": b, "flops": rows * case["experts"] * (8 if step else 4)}
    if op in ("norms", "norms_grad"):
        n = case["n"]
        params = (case["gate"] + (1, 0)[case["norm_f"] == "none"] + (case["norm_f"] == "layer") + 1
                  + (case["norm_y"] == "layer"))
        stats = sum({"none": 0, "rms": 4, "layer": 8}[case[k]] for k in ("norm_f", "norm_y"))
        if op == "norms":
            return {"bytes": 4 * rows * n * size + 4 * n * params + stats * rows, "flops": 16 * rows * n}
        return {"bytes": 6 * rows * n * size + 8 * n * params + stats * rows, "flops": 30 * rows * n}
    if op == "keep":
        values, blocks = rows * case["n"], rows * -(-case["n"] // BLOCK)
        return {"bytes": values * (3 * size + 2) + 2 * blocks, "flops": 12 * values}
    k, values = case["k"], rows * case["width"]
    if op == "dispatch":
        return {"bytes": values * size * (1 + k) + 12 * rows * k + 4 * case["experts"] + 4, "flops": 0}
    if op == "combine":
        return {"bytes": values * size * (1 + k + case["residual"]) + rows * k * (4 + 4 * case["weighted"]),
                "flops": 2 * values * k}
    return {"bytes": values * size * (1 + 2 * k) + 12 * rows * k, "flops": 3 * values * k}


# ---- the definitions in fp64 ---------------------------------------------------------

def _f64_act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu_tanh":                                   # (1 + tanh u) / 2 = 1 / (1 + exp(-2u))
        return z / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def _f64_norm(x, kind):
    """xhat, mean and 1 / deviation of each row."""
    n = x.shape[1]
    mean = x.sum(1, keepdim=True) / n if kind == "layer" else torch.zeros_like(x[:, :1])
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).sum(1, keepdim=True) / n + EPS)
    return (x - mean) * rstd, mean[:, 0], rstd[:, 0]


def _exact_router(s, case):
    l = s["logits"].double()
    rows, experts = l.shape
    index = torch.arange(experts, device=l.device)
    left, chosen = l.clone(), []
    for _ in range(case["k"]):
        best = left.max(1, keepdim=True).values
        at = torch.where(left == best, index, experts).min(1).values
        left[torch.arange(rows, device=l.device), at] = -math.inf
        chosen.append(torch.where(best[:, 0] == -math.inf, -1, at))
    ids = torch.stack(chosen, 1)
    mine = (ids[:, :, None] == index).double()               # rows x k x experts
    open_ = torch.isfinite(l) if case["over"] == "all" else mine.sum(1) > 0
    p = torch.where(open_, torch.exp(torch.where(open_, l, 0.0)), 0.0)
    p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
    out = {"ids": ids.int(), "weights": case["scale"] * torch.einsum("rke,re->rk", mine, p)}
    if case["op"] == "router_step":
        g = case["scale"] * torch.einsum("rke,rk->re", mine, s["dweights"].double())
        out["dlogits"] = p * (g - torch.einsum("re,re->r", p, g)[:, None])
    return out


def _exact_norms(s, case):
    d = {k: s[k].double() for k in ("x", "f", "s", "dy", "ds", "gate", "gamma_f", "beta_f", "gamma_y", "beta_y")
         if s.get(k) is not None}
    one = torch.ones((), dtype=torch.float64, device="cuda")
    gate, gamma_f, gamma_y = (d.get(k, one) for k in ("gate", "gamma_f", "gamma_y"))
    kind_f, kind_y = case["norm_f"], case["norm_y"]
    if case["op"] == "norms":
        out, nf = {}, d["f"]
        if kind_f != "none":
            xhat, out["mean_f"], out["rstd_f"] = _f64_norm(nf, kind_f)
            nf = xhat * gamma_f + d.get("beta_f", 0.0)
        t = case["alpha"] * d["x"] + gate * nf
        xhat, out["mean_y"], out["rstd_y"] = _f64_norm(t, kind_y)
        out.update(s=t, y=xhat * gamma_y + d.get("beta_y", 0.0))
        return {k: v for k, v in out.items() if not (k == "mean_f" and kind_f != "layer" or k == "mean_y" and kind_y != "layer")}
    st, n = s["stats"].double()[:, :, None], case["n"]

    def through(g, xhat, rstd, kind):
        less = g.sum(1, keepdim=True) / n if kind == "layer" else 0.0
        return rstd * (g - less - xhat * ((g * xhat).sum(1, keepdim=True) / n))

    yhat = (d["s"] - (st[2] if kind_y == "layer" else 0.0)) * st[3]
    t = d["ds"] + through(d["dy"] * gamma_y, yhat, st[3], kind_y)
    out = {"dx": case["alpha"] * t, "dgamma_y": torch.einsum("rn,rn->n", d["dy"], yhat)}
    if kind_y == "layer":
        out["dbeta_y"] = d["dy"].sum(0)
    fhat = d["f"] if kind_f == "none" else (d["f"] - (st[0] if kind_f == "layer" else 0.0)) * st[1]
    a, b = torch.einsum("rn,rn->n", t, fhat), t.sum(0)
    out["df"] = gate * t if kind_f == "none" else through(gate * gamma_f * t, fhat, st[1], kind_f)
    if case["gate"]:
        out["dgate"] = gamma_f * a + d.get("beta_f", 0.0) * b
    if kind_f != "none":
        out["dgamma_f"] = gate * a
    if kind_f == "layer":
        out["dbeta_f"] = gate * b
    return out


def _exact_kept(z):
    """The nearest value of a table of e4m3's, ties to the even one."""
    rows, n = z.shape
    values = [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)]
    values = torch.tensor(values[:-1], dtype=torch.float64, device=z.device)     # up to 448
    power = lambda i: ((i.long() + 1023) << 52).view(torch.float64)  # noqa: E731  (2 ** i rounds on the GPU)
    out = torch.zeros_like(z)
    for c in range(0, n, BLOCK):
        part = z[:, c:c + BLOCK]
        top = part.abs().max(1, keepdim=True).values
        e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 448.0))
        e = torch.where(top > 448.0 * power(e), e + 1, e)
        e = torch.where(top <= 448.0 * power(e - 1), e - 1, e).clamp(min=-127)
        v = part / power(e)
        up = torch.searchsorted(values, v.abs().contiguous()).clamp(max=len(values) - 1)
        low = (up - 1).clamp(min=0)
        to_up, to_low = values[up] - v.abs(), v.abs() - values[low]
        code = torch.where((to_up < to_low) | ((to_up == to_low) & (up % 2 == 0)), up, low)
        out[:, c:c + BLOCK] = torch.sign(part) * values[code] * power(e)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("router", "router_step"):
        return _exact_router(s, case)
    if op in ("norms", "norms_grad"):
        return _exact_norms(s, case)
    if op == "keep":
        z = _exact_kept(s["z"].double())
        return {"z": z, "h": _f64_act(z, case["act"])}
    rows, k, experts = case["rows"], case["k"], case["experts"]
    if op == "dispatch":
        flat = s["ids"].flatten()
        place, source, offsets = torch.full_like(flat, -1), torch.full_like(flat, -1), [0]
        e = torch.zeros(rows * k, case["width"], dtype=torch.float64, device="cuda")
        for i in range(experts):
            at = (flat == i).nonzero()[:, 0]
            where = slice(offsets[-1], offsets[-1] + len(at))
            place[at] = torch.arange(where.start, where.stop, dtype=flat.dtype, device="cuda")
            source[where] = at.int()
            e[where] = s["x"][at // k].double()
            offsets.append(where.stop)
        return {"offsets": torch.tensor(offsets, dtype=torch.int32, device="cuda"), "place": place.view(rows, k),
                "source": source, "e": e}
    f64 = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device="cuda")  # noqa: E731
    if op == "combine":
        y = f64(rows, case["width"]) if s["r"] is None else s["r"].double()
        for j in range(k):
            at = (s["place"][:, j] >= 0).nonzero()[:, 0]
            w = 1.0 if s["weights"] is None else s["weights"][at, j, None].double()
            y[at] += w * s["e"][s["place"][at, j].long()].double()
        return {"y": y}
    de, dw, dy = f64(rows * k, case["width"]), f64(rows, k), s["dy"].double()
    for j in range(k):
        at = (s["place"][:, j] >= 0).nonzero()[:, 0]
        rank = s["place"][at, j].long()
        de[rank] = s["weights"][at, j, None].double() * dy[at]
        dw[at, j] = torch.einsum("rn,rn->r", dy[at], s["e"][rank].double())
    return {"de": de, "dweights": dw}
