"""Rows that clusters share, many of them per cluster: rows follow one another
through the rings, the exchanges' two places are used in turn and the second sums of
a row go with the first of the next one.  152 SMs hold at most 76 clusters of two, 38
of four or 19 of eight, so each has at least six rows, more than a ring holds.
Against fp64, with the bounds of the other sizes; a recorded call and one over its
own inputs give the same bits."""
import pytest
import torch

import test_gpu_residual_norm as base
from expert_ops_util import gen_of
from paper_2409_02227_gb300 import goldy as G

pytestmark = pytest.mark.gpu
NONE, LAYER, RMS = base.NONE, base.LAYER, base.RMS
# clusters: backwards two; both ways two and four; four and eight; forwards eight (backwards rows stream)
SIZES = [(500, 5000), (500, 9000), (250, 20000), (130, 40000)]
# whole vectors, alike off a block, anyhow
LAYOUTS = {"whole": (0, (0, 0, 0, 0), (0, 0, 0, 0)), "framed": (-1, (0, 0, 0, 0), (3, 3, 3, 3)),
           "any": (-3, (0, 1, 2, 3), (1, 0, 3, 5))}


def case(rows, n, dtype, norm_f, norm_y, layout, **kw):
    less, more, start = LAYOUTS[layout]
    return base.Case(rows, n + less, dtype, norm_f, norm_y, more=more, start=start, **kw)


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n", SIZES)
@pytest.mark.parametrize("norm_f,norm_y", [(RMS, RMS), (LAYER, LAYER)])
def test_many_rows_per_cluster(cuda_ok, rows, n, norm_f, norm_y, dtype, layout):
    case(rows, n, dtype, norm_f, norm_y, layout).check_backward()


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("norm_f,norm_y", [(NONE, LAYER), (LAYER, NONE), (NONE, RMS), (RMS, NONE)])
def test_one_norm(cuda_ok, norm_f, norm_y, layout):
    case(300, 9000, "bf16", norm_f, norm_y, layout).check_backward(with_ds=False)


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_and_recorded(cuda_ok, dtype, layout):
    rows, n = 500, 9000
    make = lambda: case(rows, n, dtype, LAYER, RMS, layout)  # noqa: E731
    if layout == "any":                                     # a result over an input has its stride
        make = lambda: base.Case(rows, n - 3, dtype, LAYER, RMS, more=(1, 1, 1, 1), start=(1, 0, 3, 5))  # noqa: E731
    dy, ds, s, stats, dx, df, grads = make().check_backward()
    first = make()
    want_s, want_y, _ = first.check_forward()
    c = make()
    G.goldy_residual_norm_forward(c.d, c.params, c.x.ptr, c.f.ptr, c.f.ptr, c.x.ptr)
    torch.cuda.synchronize()
    assert torch.equal(c.f.t, want_s.t) and torch.equal(c.x.t, want_y.t) and c.f.guarded() and c.x.guarded()
    c = make()
    arrays = [c.new(3, dy.t), c.new(2, ds.t), c.f, c.new(2, s.t)]
    got = c.backward(arrays[0], arrays[1], arrays[3], stats, arrays[1], arrays[0])
    assert torch.equal(arrays[1].t, dx.t) and torch.equal(arrays[0].t, df.t)
    assert all(torch.equal(got[k], grads[k]) for k in grads)
    # recorded, with other inputs in the same arrays at the replay
    c = make()
    x, f = c.x.t.clone(), c.f.t.clone()
    out_s, out_y, out_stats = c.new(2), c.new(3), torch.zeros(4, rows, device="cuda")
    c.x.t.normal_(generator=gen_of(1))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        G.goldy_residual_norm_forward(c.d, c.params, c.x.ptr, c.f.ptr, out_s.ptr, out_y.ptr, out_stats.data_ptr(),
                                      torch.cuda.current_stream().cuda_stream)
    for _ in range(2):
        graph.replay()
        c.x.t.copy_(x)
        c.f.t.copy_(f)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out_s.t, want_s.t) and torch.equal(out_y.t, want_y.t)
        out_s.t.fill_(0.0), out_y.t.fill_(0.0), c.x.t.zero_()
