"""The operators around experts once more, with nothing left from an earlier run to
hide behind: every result and intermediate is overwritten before each run (NaN in
floating-point arrays, another number in the others), bounds and references have to
be numbers themselves, and the workspace has a pattern behind its last byte."""
import pytest
import torch

import test_gpu_expert_ops_order as order
import test_gpu_keep8 as keep8
import test_gpu_residual_norm as norms
import test_gpu_route as route
import test_gpu_router as router
from expert_ops_util import within
from paper_2409_02227_gb300 import goldy as G

pytestmark = pytest.mark.gpu
INPUTS = ("x", "n", "w1", "w2", "wr", "gate", "gamma")
TAIL, PATTERN = 4096, 0xA5


def spoil(chain):
    for k, t in chain.t.items():
        if k not in INPUTS:
            t.fill_(float("nan") if t.is_floating_point() else 0x5A if t.dtype == torch.uint8 else -7)
    torch.cuda.synchronize()


def results(chain):
    out = chain.results()
    del out["stats"]                                        # F's norm has no mean: row 0 is left as it was
    out["deviations"] = chain.t["stats"][1:].clone()
    assert torch.isnan(chain.t["stats"][0]).all()
    for k, t in out.items():
        if t.is_floating_point():
            assert torch.isfinite(t).all(), k               # every element has been written
        elif t.dtype == torch.int32:
            assert (t != -7).all(), k
    return out


def equal(got, want):
    for k in want:
        assert torch.equal(got[k], want[k]), k


def filled(chain, seed, **kw):
    chain.fill(seed)
    spoil(chain)
    chain.run(**kw)
    return results(chain)


@pytest.mark.parametrize("shape", order.SHAPES)
def test_back_to_back(cuda_ok, shape):
    c = order.Chain(*shape)
    for seed in range(3):
        want = filled(c, seed, wait=True)
        equal(filled(c, seed), want)
    assert G.goldy_device_error(clear=True) == 0


@pytest.mark.parametrize("shape", order.SHAPES)
def test_replayed(cuda_ok, shape):
    c = order.Chain(*shape)
    want = [filled(c, seed, wait=True) for seed in range(3)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for seed in range(3):
        c.fill(seed)
        spoil(c)
        graph.replay()
        equal(results(c), want[seed])


@pytest.mark.parametrize("shape", order.SHAPES)
def test_two_streams(cuda_ok, shape):
    """Two chains of different inputs at once, both compared."""
    chains = [order.Chain(*shape) for _ in range(2)]
    want = [filled(c, 5 + i, wait=True) for i, c in enumerate(chains)]
    streams = [torch.cuda.Stream() for _ in chains]
    for c in chains:
        spoil(c)
    for _ in range(3):
        for c, s in zip(chains, streams):
            c.run(stream=s.cuda_stream)
    for c, w in zip(chains, want):
        equal(results(c), w)


@pytest.mark.parametrize("shape", order.SHAPES[:4])
def test_partition(cuda_ok, shape):
    c = order.Chain(*shape)
    want = filled(c, 3, wait=True)
    part = G.goldy_partition_create(32, 1)
    _, (stream,) = G.goldy_partition_query(part, 1)
    spoil(c)
    c.run(stream=stream)
    equal(results(c), want)
    assert G.goldy_device_error(clear=True) == 0


@pytest.fixture
def strict(monkeypatch):
    """The operators' own tests with references and bounds that are numbers, and a
    guarded workspace of exactly the asked size."""
    made = []

    def numbers(got, ref, tol, what):
        assert torch.isfinite(ref).all(), f"{what}: reference"
        assert torch.isfinite(torch.as_tensor(tol)).all(), f"{what}: bound"
        within(got, ref, tol, what)

    def guarded(need):
        whole = torch.full((need + TAIL,), PATTERN, dtype=torch.uint8, device="cuda")
        whole[:need] = 0
        made.append((whole, need))
        return whole[:need]

    for module in (norms, route, router, keep8):
        if hasattr(module, "within"):
            monkeypatch.setattr(module, "within", numbers)
        if hasattr(module, "workspace"):
            monkeypatch.setattr(module, "workspace", guarded)
    yield made
    torch.cuda.synchronize()
    for whole, need in made:
        assert (whole[need:] == PATTERN).all(), f"written behind a workspace of {need} bytes"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n", norms.SIZES + [(40, 4096), (300, 8192), (160, 12288), (1000, 1023)])
def test_norms(cuda_ok, strict, rows, n, dtype):
    norms.Case(rows, n, dtype, norms.LAYER, norms.RMS).check_backward()
    norms.Case(rows, n, dtype, norms.RMS, norms.LAYER, more=(1, 1, 1, 1), start=(1, 1, 1, 1)).check_backward()
    assert len(strict) == 2


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("experts,k", [(2, 2), (60, 6), (256, 8), (257, 16), (1025, 8)])
def test_router(cuda_ok, strict, experts, k, dtype):
    router.test_sizes(None, 40, experts, k, dtype, router.ALL)
    router.test_sizes(None, 40, experts, k, dtype, router.CHOSEN)


@pytest.mark.parametrize("rows,k,groups", [(16, 6, 64), (512, 8, 16), (1366, 3, 60), (700, 6, 2000), (1000, 5, 4096), (160001, 4, 33)])
def test_sort(cuda_ok, strict, rows, k, groups):
    route.test_sort(None, rows, k, groups)
    assert len(strict) == 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", route.SHAPES)
def test_rows(cuda_ok, strict, shape, dtype):
    route.test_combine(None, shape, dtype, True, True)
    route.test_combine_grad(None, shape, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", keep8.ACTS)
def test_kept(cuda_ok, strict, act, dtype):
    keep8.test_act(None, act, dtype)
