"""Router, sort, dispatch, products, combine, norms and 8-bit rows back to back on
one stream, each reading what the one before has just written, over buffers that
are used again and again: the bits of the same calls with the GPU waited for after
each; of the calls inside an SM partition; and of a recorded CUDA graph."""
import pytest
import torch

from expert_ops_util import gen_of
from paper_2409_02227_gb300 import goldy as G

pytestmark = pytest.mark.gpu
F32, BF16 = G.GOLDY_F32, G.GOLDY_BF16


class Chain:
    def __init__(self, rows, width, hidden, experts, k):
        gen = gen_of(rows)
        row = lambda r, n: torch.empty(r, n, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        vec = lambda *n: torch.empty(*n, device="cuda")  # noqa: E731
        whole = lambda *n: torch.empty(*n, device="cuda", dtype=torch.int32)  # noqa: E731
        slots = rows * k
        self.router = G.router_desc(rows, experts, k, over=G.GOLDY_ROUTER_CHOSEN)
        self.route = G.route_desc(rows, k, experts, width)
        self.up = G.linear_desc(slots, width, hidden, groups=experts, act=G.GOLDY_ACT_SILU)
        self.down = G.linear_desc(slots, hidden, width, groups=experts, act_x=G.GOLDY_ACT_SILU)
        self.scores = G.linear_desc(rows, width, experts, y_dtype=F32, ldw=experts, ldy=experts)
        self.join = G.residual_norm_desc(rows, width, G.GOLDY_NORM_RMS, G.GOLDY_NORM_LAYER, alpha=0.9)
        self.kept = G.keep8_desc(slots, hidden, act=G.GOLDY_ACT_SILU)
        q, s = G.goldy_keep8_query(self.kept)
        self.t = dict(x=row(rows, width), n=row(rows, width), logits=vec(rows, experts), ids=whole(rows, k), w=vec(rows, k),
                      offsets=whole(experts + 1), place=whole(slots), source=whole(slots), e=row(slots, width), z=row(slots, hidden),
                      h=row(slots, hidden), o=row(slots, width), f=row(rows, width), s=row(rows, width), y=row(rows, width),
                      stats=vec(4, rows), q=torch.empty(q, device="cuda", dtype=torch.uint8),
                      scales=torch.empty(s, device="cuda", dtype=torch.uint8), z8=row(slots, hidden), h8=row(slots, hidden),
                      dx=row(rows, width), df=row(rows, width), do=row(slots, width), dw=vec(rows, k), dlogits=vec(rows, experts),
                      dz=row(slots, hidden), de=row(slots, width), dn=row(rows, width), dgate=vec(width), dgf=vec(width),
                      dgy=vec(width), dby=vec(width),
                      w1=(torch.randn(experts, width, hidden, generator=gen, device="cuda") * width ** -0.5).bfloat16(),
                      w2=(torch.randn(experts, hidden, width, generator=gen, device="cuda") * hidden ** -0.5).bfloat16(),
                      wr=(torch.randn(width, experts, generator=gen, device="cuda") * width ** -0.5).bfloat16(),
                      gate=1 + 0.1 * torch.randn(width, generator=gen, device="cuda"),
                      gamma=1 + 0.1 * torch.randn(width, generator=gen, device="cuda"))
        p = self.p = {k_: v.data_ptr() for k_, v in self.t.items()}
        self.params = G.residual_norm_params(gate=p["gate"], gamma_f=p["gamma"], gamma_y=p["gamma"])
        self.grads = G.residual_norm_params(gate=p["dgate"], gamma_f=p["dgf"], gamma_y=p["dgy"], beta_y=p["dby"])
        need = max([G.goldy_linear_query(d) for d in (self.up, self.down, self.scores)] +
                   [G.goldy_route_query(self.route), G.goldy_residual_norm_query(self.join)])
        self.ws = torch.zeros(max(need, 256), dtype=torch.uint8, device="cuda")
        self.fill(0)

    def fill(self, seed):
        """New inputs; rows that no expert has hold what a stale read would show."""
        gen = gen_of(seed)
        self.t["x"].normal_(generator=gen)
        self.t["n"].normal_(generator=gen)

    def run(self, wait=False, stream=None):
        p, st = self.p, torch.cuda.current_stream().cuda_stream if stream is None else stream
        kw = dict(workspace=self.ws.data_ptr(), workspace_bytes=self.ws.numel(), stream=st)
        by = dict(kw, offsets=p["offsets"])
        calls = [
            lambda: G.goldy_linear_forward(self.scores, p["n"], p["wr"], p["logits"], **kw),
            lambda: G.goldy_router_forward(self.router, p["logits"], p["ids"], p["w"], st),
            lambda: G.goldy_route_sort(self.route, p["ids"], p["offsets"], p["place"], p["source"], **kw),
            lambda: G.goldy_route_dispatch(self.route, p["n"], p["place"], p["e"], st),
            lambda: G.goldy_linear_forward(self.up, p["e"], p["w1"], p["h"], z=p["z"], **by),
            lambda: G.goldy_linear_forward(self.down, p["h"], p["w2"], p["o"], **by),
            lambda: G.goldy_keep8_pack(self.kept, p["z"], p["q"], p["scales"], st),
            lambda: G.goldy_route_combine(self.route, p["o"], p["place"], p["f"], p["w"], stream=st),
            lambda: G.goldy_residual_norm_forward(self.join, self.params, p["x"], p["f"], p["s"], p["y"], p["stats"], st),
            lambda: G.goldy_keep8_unpack(self.kept, p["q"], p["scales"], p["z8"], p["h8"], st),
            lambda: G.goldy_residual_norm_backward(self.join, self.params, p["y"], p["x"], p["f"], p["s"], p["stats"], p["dx"], p["df"],
                                                   self.grads, **kw),
            lambda: G.goldy_route_combine_grad(self.route, p["df"], p["o"], p["place"], p["w"], p["do"], p["dw"], st),
            lambda: G.goldy_router_backward(self.router, p["logits"], p["ids"], p["dw"], p["dlogits"], st),
            lambda: G.goldy_linear_input_grad(self.down, p["do"], p["w2"], p["dz"], z=p["z8"], **by),
            lambda: G.goldy_linear_input_grad(self.up, p["dz"], p["w1"], p["de"], **by),
            lambda: G.goldy_route_combine(self.route, p["de"], p["place"], p["dn"], stream=st),
            # and once more with what came out of it
            lambda: G.goldy_residual_norm_forward(self.join, self.params, p["dx"], p["dn"], p["s"], p["y"], p["stats"], st),
        ]
        for call in calls:
            call()
            if wait:
                torch.cuda.synchronize()

    def results(self):
        torch.cuda.synchronize()
        behind = int(self.t["offsets"][-1])
        out = {k: v.clone() for k, v in self.t.items()}
        for k in ("e", "z", "h", "o", "z8", "h8", "do", "dz", "de"):
            out[k] = out[k][:behind]                        # rows behind the last expert's are no result
        blocks = -(-self.kept.n // 32)
        out["q"], out["scales"] = out["q"][:behind * blocks * 32], out["scales"][:behind * blocks]
        return out


SHAPES = [(1, 64, 128, 8, 2), (60, 128, 264, 16, 4), (500, 72, 96, 31, 3), (3000, 512, 256, 64, 6), (40, 9000, 64, 4, 2)]


@pytest.mark.parametrize("shape", SHAPES)
def test_each_call_sees_the_one_before(cuda_ok, shape):
    c = Chain(*shape)
    for seed in range(4):
        c.fill(seed)
        c.run()
        together = c.results()
        c.fill(seed)
        c.run(wait=True)
        apart = c.results()
        for k in apart:
            assert torch.equal(together[k], apart[k]), k
    assert G.goldy_device_error(clear=True) == 0 and not c.ws[:65536].any()


@pytest.mark.parametrize("shape", SHAPES)
def test_replay(cuda_ok, shape):
    c = Chain(*shape)
    c.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for seed in range(3):
        c.fill(seed)
        graph.replay()
        got = c.results()
        c.fill(seed)
        c.run()
        want = c.results()
        for k in want:
            assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("shape", SHAPES)
def test_another_stream_and_workspace(cuda_ok, shape):
    """Two chains at once on streams of their own, each with its workspace."""
    a, b = Chain(*shape), Chain(*shape)
    b.fill(1)
    a.run(wait=True)
    want = a.results()
    streams = [torch.cuda.Stream() for _ in range(2)]
    a.fill(0)
    torch.cuda.synchronize()
    for _ in range(3):
        a.run(stream=streams[0].cuda_stream)
        b.run(stream=streams[1].cuda_stream)
    got = a.results()
    for k in want:
        assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("shape", SHAPES[:4])
def test_inside_a_partition(cuda_ok, shape):
    """A quarter of the SMs gives the same bits (but for rows that clusters share
    outside it, see the norms' tests)."""
    c = Chain(*shape)
    c.run(wait=True)
    want = c.results()
    part = G.goldy_partition_create(32, 1)
    sms, (stream,) = G.goldy_partition_query(part, 1)
    assert 0 < sms < 152
    c.fill(0)
    torch.cuda.synchronize()
    c.run(stream=stream)
    got = c.results()
    for k in want:
        assert torch.equal(got[k], want[k]), k
    assert G.goldy_device_error(clear=True) == 0
