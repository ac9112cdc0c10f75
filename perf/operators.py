"""Measured cases of the layer operators: a linear layer's products with the
work around them fused in (bias, activation, residual; the activation's
gradient; the bias gradient), the same products grouped by expert over ragged
row ranges, and layer norm, each forwards and backwards.

Every case runs through ``run`` in one of two forms: elementary torch
operations in fp32 (``own`` false) or the calls a user makes of the package
(``own`` true).  ``exact`` gives the same results from the definitions in
fp64.

A case is a dict of plain values:

  op        "product", "product_grad", "norm" or "norm_grad"
  rows      rows of X (tokens; all experts' together)
  fan_in, fan_out   features in and out (products)
  groups    0: one product for all rows; else that many experts with ragged,
            partly empty row ranges, given by offsets on the device
  act       product: activation of the output; product_grad: the activation
            that made X, whose gradient the input gradient is multiplied by
  bias, residual, save   product: which of them are there (save: the
            pre-activation is written out for the backward pass)
  out       type of Y, or of dW ("bf16" or "f32")
  n, dtype  norm: features and type of X, Y and their gradients
"""
from __future__ import annotations

import math
import random

import torch

own = False

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SKIPPED_SIZES = (3072,)      # never drawn
MOST_FLOPS = 2.0 * 8192 * 2048 * 4096
MOST_WEIGHTS = 16 * 2048 * 4096
MOST_NORM = 16384 * 4096
EPS = 1e-5


def product(name, rows, fan_in, fan_out, groups=0, act="none", bias=True, residual=False, save=False, out="bf16"):
    return {"name": name, "op": "product", "rows": rows, "fan_in": fan_in, "fan_out": fan_out, "groups": groups,
            "act": act, "bias": bias, "residual": residual, "save": save, "out": out}


def product_grad(name, rows, fan_in, fan_out, groups=0, act="none", out="f32"):
    return {"name": name, "op": "product_grad", "rows": rows, "fan_in": fan_in, "fan_out": fan_out,
            "groups": groups, "act": act, "out": out}


def norm(name, op, rows, n, dtype="bf16"):
    return {"name": name, "op": op, "rows": rows, "n": n, "dtype": dtype}


def listed():
    return [
        # one token through a layer: weights are read once, latency counts
        product("product_token", 1, 1024, 4096, act="silu"),
        # a small serving batch through a down projection, residual added
        product("product_batch", 37, 4096, 1024, residual=True),
        # the first layer of a feed-forward block in training: the
        # pre-activation is kept for the backward pass
        product("product_train", 2048, 2048, 8192, act="gelu", save=True),
        # odd sizes with padded strides, fp32 out (a head or a probe)
        product("product_odd_f32", 1999, 1000, 1357, act="gelu_tanh", residual=True, out="f32"),
        # the second layer's backward pass: input gradient through the
        # activation, weight gradient, bias gradient
        product_grad("product_grad", 2048, 8192, 2048, act="gelu"),
        # decoding: 32 rows over 8 experts, some without any
        product("experts_decode", 32, 1024, 4096, groups=8, act="silu"),
        # a prompt over 16 experts in training form
        product("experts_prompt", 8192, 2048, 4096, groups=16, act="gelu", save=True),
        # the experts' backward pass
        product_grad("experts_grad", 8192, 2048, 1024, groups=8, act="silu", out="bf16"),
        # one token's norm: latency only
        norm("norm_token", "norm", 1, 4096),
        # a training batch
        norm("norm_train", "norm", 16384, 4096),
        norm("norm_grad", "norm_grad", 16384, 2048),
        # fp32 with an odd row length: rows start off a vector's boundary
        norm("norm_grad_odd_f32", "norm_grad", 1000, 1023, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A feature count: half of the time a multiple of 64, else any."""
    while True:
        v = _log(rng, lo, hi)
        if rng.random() < 0.5:
            v = max(lo, 64 * round(v / 64))
        if v not in SKIPPED_SIZES:
            return v


def draw(rng):
    op = rng.choice(["product", "product", "product_grad", "norm", "norm_grad"])
    if op in ("norm", "norm_grad"):
        while True:
            rows, n = _log(rng, 1, 16384), _size(rng, 16, 8192)
            if rows * n <= MOST_NORM // (2 if op == "norm_grad" else 1):
                return {"op": op, "rows": rows, "n": n, "dtype": rng.choice(["bf16", "bf16", "f32"])}
    groups = rng.choice([0, 0, 0, 4, 8, 16, 31, 64])
    while True:
        rows, fan_in, fan_out = _log(rng, 1, 8192), _size(rng, 64, 8192), _size(rng, 64, 8192)
        flops = 2.0 * rows * fan_in * fan_out * (2 if op == "product_grad" else 1)
        if flops <= MOST_FLOPS and max(groups, 1) * fan_in * fan_out <= MOST_WEIGHTS:
            break
    case = {"op": op, "rows": rows, "fan_in": fan_in, "fan_out": fan_out, "groups": groups,
            "act": rng.choice(ACTS), "out": rng.choice(["bf16", "f32"])}
    if op == "product":
        case.update(bias=rng.random() < 0.7, residual=rng.random() < 0.5, save=rng.random() < 0.4)
    return case


# ---- inputs -------------------------------------------------------------------

def _matrix(gen, rows, cols, scale=1.0, lead=()):
    """A bf16 matrix (or a stack of them) whose rows start on 16-byte
    boundaries, as the products need them: padded where the width is odd."""
    ld = (cols + 7) // 8 * 8
    t = torch.empty(*lead, rows, ld, device="cuda", dtype=torch.bfloat16)
    step = max(1, (1 << 27) // max(1, t[..., 0].numel() // max(1, rows) * ld))    # rows per chunk of fp32 values
    for r in range(0, rows, step):
        part = t[..., r:r + step, :]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda") * scale)
    return t[..., :cols]


def _counts(case, seed):
    """Rows of each expert: an uneven router, one expert in eight unused."""
    groups, rows = case["groups"], case["rows"]
    rng = random.Random(seed * 7919 + 1)
    weight = [0.0 if rng.random() < 0.125 else math.exp(rng.gauss(0.0, 0.5)) for _ in range(groups)]
    if not any(weight):
        weight[0] = 1.0
    counts = [0] * groups
    for e in rng.choices(range(groups), weight, k=rows):
        counts[e] += 1
    return counts


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    rows = case["rows"]
    if case["op"] in ("norm", "norm_grad"):
        n, dtype = case["n"], TYPES[case["dtype"]]
        # a residual stream: a few features stand out, and the mean is not 0
        feature = torch.randn(n, generator=gen, device="cuda")
        scale = 1.0 + 4.0 * (torch.rand(n, generator=gen, device="cuda") < 0.02)
        s["x"] = (torch.randn(rows, n, generator=gen, device="cuda") * scale + 0.3 * feature + 0.1).to(dtype)
        s["gamma"] = (1.0 + 0.1 * torch.randn(n, generator=gen, device="cuda")).to(dtype)
        s["beta"] = (0.1 * torch.randn(n, generator=gen, device="cuda")).to(dtype)
        if case["op"] == "norm_grad":
            s["dy"] = (0.01 * torch.randn(rows, n, generator=gen, device="cuda")).to(dtype)
            x = s["x"].double()
            s["mean"] = x.mean(1).float()
            s["rstd"] = torch.rsqrt(x.var(1, unbiased=False) + EPS).float()
    else:
        fan_in, fan_out, groups = case["fan_in"], case["fan_out"], case["groups"]
        lead = (groups,) if groups else ()
        s["w"] = _matrix(gen, fan_in, fan_out, fan_in ** -0.5, lead)
        if groups:
            counts = _counts(case, seed)
            s["counts"] = counts
            starts = [sum(counts[:e]) for e in range(groups + 1)]
            s["offsets"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
            most = max(counts)
            e = torch.repeat_interleave(torch.arange(groups), torch.tensor(counts))
            at = e * most + (torch.arange(rows) - torch.tensor(starts)[e])
            padded = torch.full((groups * most,), rows)
            padded[at] = torch.arange(rows)
            s["at"], s["padded"] = at.cuda(), padded.view(groups, most).cuda()
        if case["op"] == "product":
            s["x"] = _matrix(gen, rows, fan_in)
            if case["bias"]:
                s["b"] = (0.1 * torch.randn(*lead, fan_out, generator=gen, device="cuda")).bfloat16()
            if case["residual"]:
                r = _matrix(gen, rows, fan_out)
                s["r"] = r if case["out"] == "bf16" else r.float()
        else:
            s["z"] = _matrix(gen, rows, fan_in)
            s["x"] = s["z"].clone(memory_format=torch.preserve_format) if case["act"] == "none" else _matrix(gen, rows, fan_in)
            if case["act"] != "none":
                s["x"].copy_(_act(s["z"].float(), case["act"]))
            s["dy"] = _matrix(gen, rows, fan_out, 0.01)
    if own:
        _plan(s)
    return s


# ---- the calls a user makes -----------------------------------------------------

def _plan(s):
    """What a user's program keeps: descriptors, output buffers, a workspace."""
    from paper_2409_02227_gb300 import goldy as G

    case, rows = s["case"], s["case"]["rows"]
    bf16, f32 = G.GOLDY_BF16, G.GOLDY_F32
    kind = {"bf16": bf16, "f32": f32}
    empty = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    padded = lambda cols, dtype: empty(rows, (cols + 7) // 8 * 8, dtype=dtype)[:, :cols]  # noqa: E731
    if case["op"] in ("norm", "norm_grad"):
        n = case["n"]
        s["desc"] = d = G.layernorm_desc(rows, n, dtype=kind[case["dtype"]], param_dtype=kind[case["dtype"]], eps=EPS)
        if case["op"] == "norm":
            s["y"] = torch.empty_like(s["x"])
            s["mean"], s["rstd"] = empty(rows, dtype=torch.float32), empty(rows, dtype=torch.float32)
        else:
            s["dx"] = torch.empty_like(s["x"])
            s["dgamma"], s["dbeta"] = empty(n, dtype=torch.float32), empty(n, dtype=torch.float32)
        need = G.goldy_layernorm_query(d)
    else:
        fan_in, fan_out, groups = case["fan_in"], case["fan_out"], case["groups"]
        act = getattr(G, "GOLDY_ACT_" + case["act"].upper())
        ldx, ldw = s["x"].stride(0), s["w"].stride(-2)
        lead = (groups,) if groups else ()
        if case["op"] == "product":
            s["y"] = padded(fan_out, TYPES[case["out"]])
            if case["save"]:
                s["z"] = padded(fan_out, torch.bfloat16)
            s["desc"] = d = G.linear_desc(rows, fan_in, fan_out, groups=groups, act=act, y_dtype=kind[case["out"]],
                                          bias_dtype=bf16, ldx=ldx, ldw=ldw, ldy=s["y"].stride(0))
        else:
            s["dx"] = padded(fan_in, torch.bfloat16)
            s["dw"] = empty(*lead, fan_in, ldw, dtype=TYPES[case["out"]])[..., :fan_out]
            s["db"] = empty(*lead, fan_out, dtype=torch.float32)
            s["desc"] = d = G.linear_desc(rows, fan_in, fan_out, groups=groups, act_x=act, dw_dtype=kind[case["out"]],
                                          ldx=ldx, ldw=ldw, ldy=s["dy"].stride(0))
        need = G.goldy_linear_query(d)
    s["work"] = torch.zeros(max(need, 256), dtype=torch.uint8, device="cuda")
    s["G"] = G


def _ptr(s, name):
    t = s.get(name)
    return 0 if t is None else t.data_ptr()


def _run_own(s):
    G, d, op = s["G"], s["desc"], s["case"]["op"]
    stream = torch.cuda.current_stream().cuda_stream
    work = (s["work"].data_ptr(), s["work"].numel())
    if op == "norm":
        G.goldy_layernorm_forward(d, _ptr(s, "x"), _ptr(s, "gamma"), _ptr(s, "beta"), _ptr(s, "y"), _ptr(s, "mean"),
                                  _ptr(s, "rstd"), stream)
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if op == "norm_grad":
        G.goldy_layernorm_backward(d, _ptr(s, "dy"), _ptr(s, "x"), _ptr(s, "gamma"), _ptr(s, "mean"), _ptr(s, "rstd"),
                                   _ptr(s, "dx"), _ptr(s, "dgamma"), _ptr(s, "dbeta"), *work, stream)
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    offsets = _ptr(s, "offsets")
    if op == "product":
        G.goldy_linear_forward(d, _ptr(s, "x"), _ptr(s, "w"), _ptr(s, "y"), bias=_ptr(s, "b"), residual=_ptr(s, "r"),
                               z=_ptr(s, "z"), offsets=offsets, workspace=work[0], workspace_bytes=work[1],
                               stream=stream)
        return {k: s[k] for k in ("y", "z") if k in s}
    z = _ptr(s, "z") if s["case"]["act"] != "none" else 0
    G.goldy_linear_input_grad(d, _ptr(s, "dy"), _ptr(s, "w"), _ptr(s, "dx"), z=z, offsets=offsets, workspace=work[0],
                              workspace_bytes=work[1], stream=stream)
    G.goldy_linear_weight_grad(d, _ptr(s, "x"), _ptr(s, "dy"), _ptr(s, "dw"), offsets=offsets, workspace=work[0],
                               workspace_bytes=work[1], stream=stream)
    G.goldy_linear_bias_grad(d, _ptr(s, "dy"), _ptr(s, "db"), offsets=offsets, workspace=work[0],
                             workspace_bytes=work[1], stream=stream)
    return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}


# ---- the plain form ---------------------------------------------------------------

def _phi(z):
    return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, 0.0, z)
    if act == "gelu":
        return z * _phi(z)
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return _phi(z) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        g = torch.sigmoid(z)
        return g * (1.0 + z * (1.0 - g))
    return torch.ones_like(z)


def _pad(s, t):
    """Rows grouped into [experts, most rows, features], zeros behind."""
    t = t.float()
    return torch.cat([t, t.new_zeros(1, t.shape[1])])[s["padded"]]


def _unpad(s, t):
    return t.reshape(-1, t.shape[-1])[s["at"]]


def _run_plain(s):
    case, op = s["case"], s["case"]["op"]
    if op == "norm":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        c = x - mean
        rstd = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
        y = c * rstd * s["gamma"].float() + s["beta"].float()
        return {"y": y.to(s["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if op == "norm_grad":
        dy = s["dy"].float()
        rstd = s["rstd"][:, None]
        xhat = (s["x"].float() - s["mean"][:, None]) * rstd
        g = dy * s["gamma"].float()
        dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * xhat).sum(0), "dbeta": dy.sum(0)}
    w, grouped = s["w"].float(), case["groups"] > 0
    if op == "product":
        if grouped:
            z = torch.bmm(_pad(s, s["x"]), w)
            z = _unpad(s, z + s["b"].float()[:, None] if "b" in s else z)
        else:
            z = s["x"].float() @ w
            z = z + s["b"].float() if "b" in s else z
        y = _act(z, case["act"])
        y = y + s["r"].float() if "r" in s else y
        out = {"y": y.to(TYPES[case["out"]])}
        return dict(out, z=z.bfloat16()) if case["save"] else out
    if grouped:
        dy, x = _pad(s, s["dy"]), _pad(s, s["x"])
        dx = _unpad(s, torch.bmm(dy, w.transpose(1, 2)))
        dw, db = torch.bmm(x.transpose(1, 2), dy), dy.sum(1)
    else:
        dy, x = s["dy"].float(), s["x"].float()
        dx, dw, db = dy @ w.t(), x.t() @ dy, dy.sum(0)
    if case["act"] != "none":
        dx = dx * _act_grad(s["z"].float(), case["act"])
    return {"dx": dx.bfloat16(), "dw": dw.to(TYPES[case["out"]]), "db": db}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ---------------------------------------------------

def work(case):
    """Each input read once and each output written once.  Of an expert's
    weights only those that some row needs count where there are fewer rows
    than experts (the weight gradient writes all of them)."""
    rows = case["rows"]
    if case["op"] in ("norm", "norm_grad"):
        n, size = case["n"], 2 if case["dtype"] == "bf16" else 4
        if case["op"] == "norm":
            return {"bytes": 2 * rows * n * size + 2 * n * size + 8 * rows, "flops": 8 * rows * n}
        return {"bytes": 3 * rows * n * size + n * size + 8 * n + 8 * rows, "flops": 14 * rows * n}
    fan_in, fan_out = case["fan_in"], case["fan_out"]
    groups = max(1, case["groups"])
    size = 2 if case["out"] == "bf16" else 4
    weights = min(groups, rows) * fan_in * fan_out
    if case["op"] == "product":
        b = 2 * rows * fan_in + 2 * weights + size * rows * fan_out
        b += 2 * min(groups, rows) * fan_out * case["bias"] + size * rows * fan_out * case["residual"]
        return {"bytes": b + 2 * rows * fan_out * case["save"], "flops": 2 * rows * fan_in * fan_out}
    b = 2 * rows * fan_out + 2 * weights + 2 * rows * fan_in + 2 * rows * fan_in + size * groups * fan_in * fan_out
    b += 2 * rows * fan_in * (case["act"] != "none") + 4 * groups * fan_out
    return {"bytes": b, "flops": 4 * rows * fan_in * fan_out}


# ---- the definitions in fp64 ---------------------------------------------------------

def _f64_act(z, act):
    """(value, derivative) of an activation."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        g = 1.0 / (1.0 + torch.exp(-z))
        return z * g, g + z * g * (1.0 - g)
    u = math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)      # gelu by tanh: (1 + tanh u) / 2 = 1 / (1 + exp(-2u))
    g = 1.0 / (1.0 + torch.exp(-2.0 * u))
    return z * g, g + z * 2.0 * g * (1.0 - g) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * z ** 2)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm", "norm_grad"):
        x, n = s["x"].double(), case["n"]
        if case["op"] == "norm":
            mean = x.sum(1) / n
            var = ((x - mean[:, None]) ** 2).sum(1) / n
            rstd = 1.0 / torch.sqrt(var + EPS)
            y = (x - mean[:, None]) * rstd[:, None] * s["gamma"].double() + s["beta"].double()
            return {"y": y, "mean": mean, "rstd": rstd}
        mean, rstd, dy = s["mean"].double()[:, None], s["rstd"].double()[:, None], s["dy"].double()
        xhat = (x - mean) * rstd
        g = dy * s["gamma"].double()
        dx = rstd * (g - g.sum(1, keepdim=True) / n - xhat * ((g * xhat).sum(1, keepdim=True) / n))
        return {"dx": dx, "dgamma": torch.einsum("rn,rn->n", dy, xhat), "dbeta": dy.sum(0)}
    rows, fan_in, fan_out, groups = case["rows"], case["fan_in"], case["fan_out"], case["groups"]
    f64 = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device="cuda")  # noqa: E731
    spans, r = [], 0
    for e, count in enumerate(s["counts"] if groups else [rows]):
        spans.append((e, slice(r, r + count)))
        r += count
    weight = lambda e: (s["w"][e] if groups else s["w"]).double()  # noqa: E731
    if case["op"] == "product":
        z = f64(rows, fan_out)
        for e, at in spans:
            z[at] = s["x"][at].double() @ weight(e)
            if case["bias"]:
                z[at] += (s["b"][e] if groups else s["b"]).double()
        y = _f64_act(z, case["act"])[0]
        if case["residual"]:
            y = y + s["r"].double()
        return {"y": y, "z": z} if case["save"] else {"y": y}
    dx, dw, db = f64(rows, fan_in), f64(max(1, groups), fan_in, fan_out), f64(max(1, groups), fan_out)
    for e, at in spans:
        dy = s["dy"][at].double()
        dx[at] = (dy @ weight(e).T) * _f64_act(s["z"][at].double(), case["act"])[1]
        dw[e] = s["x"][at].double().T @ dy
        db[e] = dy.sum(0)
    return {"dx": dx, "dw": dw, "db": db} if groups else {"dx": dx, "dw": dw[0], "db": db[0]}
