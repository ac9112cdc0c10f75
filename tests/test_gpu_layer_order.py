"""Layer calls back to back on one stream, each reading what the one before has
just written: statistics, saved pre-activations, residuals, dZ, offsets' rows.  The
buffers are used again and again for new inputs, so that a value read too early, or
from a cache that an earlier round filled, shows.  The results have to be the bits
of the same calls with the GPU waited for after each.
"""
import pytest
import torch

from paper_2409_02227_gb300 import goldy as G
from test_gpu_linear import ACTS, F32, gen_of, matrix, offsets_of, ptr

pytestmark = pytest.mark.gpu


def chain(s, wait):
    """A pre-norm layer forwards and backwards, its residual added in place."""
    st = torch.cuda.current_stream().cuda_stream
    kw = dict(offsets=ptr(s["offsets"]), workspace=ptr(s["ws"]), workspace_bytes=s["ws"].numel(), stream=st)
    p = {k: ptr(v) for k, v in s.items() if torch.is_tensor(v)}
    calls = [
        # gamma and beta come from a norm of their own, so from the call before
        lambda: G.goldy_layernorm_forward(s["params"], p["raw"], 0, 0, p["affine"], 0, 0, st),
        lambda: G.goldy_layernorm_forward(s["norm"], p["x"], p["affine"], p["affine"] + 4 * s["affine"].stride(0),
                                          p["n"], p["mean"], p["rstd"], st),
        lambda: G.goldy_linear_forward(s["up"], p["n"], p["w1"], p["h"], bias=p["b"], z=p["z"], **kw),
        lambda: G.goldy_linear_forward(s["down"], p["h"], p["w2"], p["y"], residual=p["n"], **kw),
        lambda: G.goldy_linear_forward(s["down"], p["h"], p["w2"], p["y"], residual=p["y"], **kw),
        lambda: G.goldy_linear_input_grad(s["down"], p["y"], p["w2"], p["dz"], z=p["z"], **kw),
        lambda: G.goldy_linear_bias_grad(s["up"], p["dz"], p["db"], **kw),
        lambda: G.goldy_linear_weight_grad(s["up"], p["n"], p["dz"], p["dw"], **kw),
        lambda: G.goldy_linear_input_grad(s["up"], p["dz"], p["w1"], p["dn"], residual=p["y"], **kw),
        lambda: G.goldy_layernorm_backward(s["norm"], p["dn"], p["x"], p["affine"], p["mean"], p["rstd"], p["dx"],
                                           p["dg"], p["dbeta"], p["ws"], s["ws"].numel(), st),
        lambda: G.goldy_layernorm_forward(s["norm"], p["dx"], p["dg"], p["dbeta"], p["n2"], p["mean"], p["rstd"], st),
        lambda: G.goldy_layernorm_backward(s["norm"], p["n2"], p["dx"], p["dg"], p["mean"], p["rstd"], p["dx2"],
                                           p["dg2"], p["dbeta2"], p["ws"], s["ws"].numel(), st),
    ]
    for call in calls:
        call()
        if wait:
            torch.cuda.synchronize()
    return {k: s[k].clone() for k in ("n", "mean", "rstd", "h", "z", "y", "dz", "db", "dw", "dn", "dx", "dg", "dbeta", "n2",
                                      "dx2", "dg2", "dbeta2")}


@pytest.mark.parametrize("rows,width,hidden,counts", [(1, 256, 512, None), (40, 128, 264, None), (300, 512, 1024, None),
                                                      (200, 136, 256, [30, 0, 100, 70]), (3000, 1024, 512, None),
                                                      (60, 9000, 64, None)])
def test_each_call_sees_the_one_before(cuda_ok, rows, width, hidden, counts):
    gen, groups = gen_of(rows), len(counts or [])
    lead = (groups,) if groups else ()
    row = lambda n, dtype=torch.bfloat16: torch.empty(rows, n, device="cuda", dtype=dtype)  # noqa: E731
    vec = lambda *n: torch.empty(*n, device="cuda")  # noqa: E731
    s = dict(norm=G.layernorm_desc(rows, width, param_dtype=F32),
             params=G.layernorm_desc(2, width, dtype=F32),
             up=G.linear_desc(rows, width, hidden, groups=groups, act=ACTS["gelu"]),
             down=G.linear_desc(rows, hidden, width, groups=groups, act_x=ACTS["gelu"]),
             offsets=offsets_of(counts), raw=vec(2, width), affine=vec(2, width), x=row(width), n=row(width), n2=row(width),
             y=row(width), dn=row(width), dx=row(width), dx2=row(width), h=row(hidden), z=row(hidden), dz=row(hidden),
             mean=vec(rows), rstd=vec(rows), dw=vec(*lead, width, hidden), db=vec(*lead, hidden),
             dg=vec(width), dbeta=vec(width), dg2=vec(width), dbeta2=vec(width),
             w1=matrix(gen, width, hidden, None, width ** -0.5, lead), w2=matrix(gen, hidden, width, None, hidden ** -0.5, lead),
             b=torch.randn(*lead, hidden, generator=gen, device="cuda").bfloat16())
    need = max(G.goldy_linear_query(s["up"]), G.goldy_linear_query(s["down"]), G.goldy_layernorm_query(s["norm"]))
    s["ws"] = torch.zeros(max(need, 256), dtype=torch.uint8, device="cuda")
    for _ in range(6):
        s["x"].copy_(torch.randn(rows, width, generator=gen, device="cuda"))
        s["raw"].copy_(torch.randn(2, width, generator=gen, device="cuda"))
        together = chain(s, False)
        apart = chain(s, True)
        for k in apart:
            assert torch.equal(together[k], apart[k]), k
    assert G.goldy_device_error(clear=True) == 0
