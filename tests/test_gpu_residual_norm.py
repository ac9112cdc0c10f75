"""The norms around a block with gate and residual scale, against fp64.

Bounds.  Every fp32 operation is off by at most u of its result, so an error is
at most (operations in a row) * u of the formula with every term replaced by its
size.  A sum over a row has at most n / 32 + 60 steps (a thread's elements, lanes,
warps, CTAs); a result lies behind two such sums forwards and behind two
backwards, and less than 60 single operations.  A gradient of a parameter is a
sum over the rows of such terms, rows / 8 + 200 steps more (a team's rows, teams,
CTAs).  A result is then rounded once to its type."""
import pytest
import torch

from expert_ops_util import HALF, TYPES, U, Rows, gen_of, within, workspace
from paper_2409_02227_gb300 import goldy as G

pytestmark = pytest.mark.gpu
NONE, LAYER, RMS = G.GOLDY_NORM_NONE, G.GOLDY_NORM_LAYER, G.GOLDY_NORM_RMS
EPS = 1e-5
NAMES = ("gate", "gamma_f", "beta_f", "gamma_y", "beta_y")


def steps(n):
    return 2 * (n / 32 + 60) + 60


def norm64(v, kind, gamma, beta, stats=None):
    """(result, size of its terms, mean, rstd)"""
    if kind == NONE:
        return v, v.abs(), None, None
    mean = v.mean(1, keepdim=True) if kind == LAYER else torch.zeros_like(v[:, :1])
    rstd = 1 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + EPS)
    xhat = (v - mean) * rstd
    size = (v.abs() + v.abs().mean(1, keepdim=True)) * rstd + xhat.abs()
    return xhat * gamma + beta, size * gamma.abs() + beta.abs(), mean[:, 0], rstd[:, 0]


class Case:
    def __init__(self, rows, n, dtype, norm_f, norm_y, given=NAMES, param="f32", alpha=0.75, more=(0, 0, 0, 0), start=(0, 0, 0, 0),
                 far=0.0, seed=0):
        gen, t = gen_of(rows + n + seed), TYPES[dtype][0]
        rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
        self.stream = 0
        self.rows, self.n, self.t, self.norm_f, self.norm_y, self.alpha = rows, n, t, norm_f, norm_y, alpha
        self.ld, self.start = [n + m for m in more], start
        self.x, self.f = self.new(0, rnd(rows, n) + far), self.new(1, 0.5 * rnd(rows, n) + 0.3 * rnd(n) + far)
        self.p = {}
        for name in NAMES:
            absent = name not in given or (name[-1] == "f" and norm_f == NONE) or (name[-1] == "y" and norm_y == NONE)
            if not absent:
                v = {"gate": 0.5, "gamm": 1.0, "beta": 0.0}[name[:4]] + 0.2 * rnd(n)
                self.p[name] = v.to(TYPES[param][0])
        self.params = G.residual_norm_params(**{k: v.data_ptr() for k, v in self.p.items()})
        self.d = G.residual_norm_desc(rows, n, norm_f, norm_y, dtype=TYPES[dtype][1], param_dtype=TYPES[param][1], eps=EPS,
                                      alpha=alpha, ldx=self.ld[0], ldf=self.ld[1], lds=self.ld[2], ldy=self.ld[3])
        self.alpha = self.d.alpha                           # as fp32 holds it
        one, zero = torch.ones(n, device="cuda", dtype=torch.float64), torch.zeros(n, device="cuda", dtype=torch.float64)
        self.v = {k: self.p[k].double() if k in self.p else (zero if k[:4] == "beta" else one) for k in NAMES}

    def new(self, which, fill=None):
        return Rows(self.rows, self.n, self.t, self.ld[which], self.start[which], fill)

    def forward64(self, x, f):
        v = self.v
        nf, size_f, mf, rf = norm64(f, self.norm_f, v["gamma_f"], v["beta_f"])
        s = self.alpha * x + v["gate"] * nf
        size_s = (self.alpha * x).abs() + v["gate"].abs() * size_f
        y, size_y, my, ry = norm64(s, self.norm_y, v["gamma_y"], v["beta_y"])
        if self.norm_y != NONE:                             # an error of S reaches Y through S, the mean and the deviation
            rms = size_s.square().mean(1, keepdim=True).sqrt()
            xhat = (s - my[:, None]) * ry[:, None]
            size_y = size_y + (size_s + rms * (1 + xhat.abs())) * ry[:, None] * v["gamma_y"].abs()
        return s, size_s, y, size_y, (mf, rf, my, ry)

    def check_forward(self):
        s, y = self.new(2), self.new(3)
        stats = torch.full((4, self.rows), 55.0, device="cuda")
        torch.cuda.synchronize()                            # the call may go to another stream
        G.goldy_residual_norm_forward(self.d, self.params, self.x.ptr, self.f.ptr, s.ptr, y.ptr if self.norm_y else 0, stats.data_ptr(),
                                      self.stream)
        torch.cuda.synchronize()
        rs, size_s, ry, size_y, want = self.forward64(self.x.t.double(), self.f.t.double())
        k = steps(self.n) * U
        within(s.t, rs, HALF[self.t] * rs.abs() + k * size_s, "S")
        if self.norm_y:
            within(y.t, ry, HALF[self.t] * ry.abs() + k * size_y, "Y")
        assert s.guarded() and y.guarded() and self.x.guarded() and self.f.guarded()
        for i, (kind, first) in enumerate(((self.norm_f, self.f.t.double()), (self.norm_y, rs))):
            size = first.abs() if i == 0 else size_s
            if kind == LAYER:
                within(stats[2 * i], want[2 * i], k * size.mean(1), f"mean {i}")
            else:
                assert (stats[2 * i] == 55.0).all()
            if kind != NONE:
                # of the deviation: an error of v by k size shifts the sum of squares by 2 |v - mean| k size
                r = want[2 * i + 1]
                c = first - (want[2 * i][:, None] if kind == LAYER else 0.0)
                off = k * (1 + r * r * (c.abs() * size).mean(1)) * r
                within(stats[2 * i + 1], r, off, f"rstd {i}")
            else:
                assert (stats[2 * i + 1] == 55.0).all()
        return s, y, stats

    def gradients64(self, dy, ds, f, s, stats):
        """The definition with the size of every term beside it."""
        v, n = self.v, self.n

        def through(g, size, x, kind, mean, rstd):
            if kind == NONE:
                return g, size, x, x.abs()
            xhat, hat = (x - mean) * rstd, (x.abs() + mean.abs()) * rstd
            d = g - xhat * (g * xhat).mean(1, keepdim=True)
            e = size + hat * (size * hat).mean(1, keepdim=True)
            if kind == LAYER:
                d, e = d - g.mean(1, keepdim=True), e + size.mean(1, keepdim=True)
            return rstd * d, rstd * e, xhat, hat

        st = stats.double()[:, :, None]
        t, size_t, out = ds, ds.abs(), {}
        if self.norm_y != NONE:
            g = dy * v["gamma_y"]
            back, size, yhat, hat = through(g, g.abs(), s, self.norm_y, st[2] if self.norm_y == LAYER else 0 * st[2], st[3])
            t, size_t = t + back, size_t + size
            out["gamma_y"], out["beta_y"] = ((dy * yhat).sum(0), (dy.abs() * hat).sum(0)), (dy.sum(0), dy.abs().sum(0))
        u, size_u = t * v["gate"] * v["gamma_f"], size_t * (v["gate"] * v["gamma_f"]).abs()
        df, size_df, fhat, hat = through(u, size_u, f, self.norm_f, st[0] if self.norm_f == LAYER else 0 * st[0], st[1])
        a, size_a, b, size_b = (t * fhat).sum(0), (size_t * hat).sum(0), t.sum(0), size_t.sum(0)
        out["gate"] = (v["gamma_f"] * a + v["beta_f"] * b, v["gamma_f"].abs() * size_a + v["beta_f"].abs() * size_b)
        if self.norm_f != NONE:
            out["gamma_f"], out["beta_f"] = (v["gate"] * a, v["gate"].abs() * size_a), (v["gate"] * b, v["gate"].abs() * size_b)
        return (self.alpha * t, abs(self.alpha) * size_t), (df, size_df), out

    def backward(self, dy, ds, s, stats, dx, df, wanted=None, accumulate=False, grads=None):
        names = [k for k in NAMES if not (k[-1] == "f" and self.norm_f == NONE or k[-1] == "y" and self.norm_y == NONE)]
        grads = {k: torch.full((self.n,), 3.0, device="cuda") for k in (names if wanted is None else wanted)}
        need = G.goldy_residual_norm_query(self.d)
        ws = workspace(need)
        torch.cuda.synchronize()
        G.goldy_residual_norm_backward(self.d, self.params, dy.ptr if self.norm_y else 0, ds.ptr if ds else 0, self.f.ptr, s.ptr,
                                       stats.data_ptr(), dx.ptr, df.ptr,
                                       G.residual_norm_params(**{k: g.data_ptr() for k, g in grads.items()}) if grads else None,
                                       ws.data_ptr() if grads else 0, need if grads else 0, self.stream, accumulate)
        torch.cuda.synchronize()
        assert not ws[:65536].any()
        return grads

    def check_backward(self, with_ds=True, wanted=None, accumulate=False):
        s, y, stats = self.check_forward()
        gen = gen_of(99 + self.n)
        rnd = lambda: torch.randn(self.rows, self.n, generator=gen, device="cuda")  # noqa: E731
        dy, ds = self.new(3, rnd()), self.new(2, rnd()) if with_ds or not self.norm_y else None
        dx, df = self.new(0), self.new(1)
        grads = self.backward(dy, ds, s, stats, dx, df, wanted, accumulate)
        zero = torch.zeros_like(s.t, dtype=torch.float64)
        rdx, rdf, rg = self.gradients64(dy.t.double(), ds.t.double() if ds else zero, self.f.t.double(), s.t.double(), stats)
        k = steps(self.n) * U
        within(dx.t, rdx[0], HALF[self.t] * rdx[0].abs() + k * rdx[1], "dX")
        within(df.t, rdf[0], HALF[self.t] * rdf[0].abs() + k * rdf[1], "dF")
        kg = (steps(self.n) + self.rows / 8 + 200) * U
        for name, g in grads.items():
            before = 3.0 if accumulate else 0.0
            within(g, rg[name][0] + before, kg * (rg[name][1] + before), "d" + name)
        assert dx.guarded() and df.guarded()
        return dy, ds, s, stats, dx, df, grads


SIZES = [(1, 1), (3, 7), (5, 16), (1, 4096), (37, 100), (700, 64), (64, 256), (50, 513), (100, 1023), (33, 2048), (300, 1000),
         (20, 4097), (9, 5000), (40, 8192), (5, 12288), (3, 20000), (2, 40000), (2, 70001)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n", SIZES)
@pytest.mark.parametrize("norm_f,norm_y", [(RMS, RMS), (LAYER, LAYER), (NONE, RMS)])
def test_sizes(cuda_ok, rows, n, norm_f, norm_y, dtype):
    Case(rows, n, dtype, norm_f, norm_y).check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm_f", [NONE, LAYER, RMS])
@pytest.mark.parametrize("norm_y", [NONE, LAYER, RMS])
def test_kinds(cuda_ok, norm_f, norm_y, dtype):
    for rows, n in ((61, 300), (17, 6000)):
        for given in (NAMES, (), ("gate",), ("gamma_f", "gamma_y")):
            Case(rows, n, dtype, norm_f, norm_y, given).check_backward()
        Case(rows, n, dtype, norm_f, norm_y, param="bf16", alpha=1.0).check_backward(with_ds=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [64, 255, 2000, 4000, 9000])
@pytest.mark.parametrize("more,start", [((8, 16, 0, 24), (8, 0, 16, 8)), ((0, 1, 2, 3), (1, 2, 3, 5)), ((1, 1, 1, 1), (0, 0, 0, 0)),
                                        ((0, 0, 0, 0), (1, 0, 0, 0)), ((0, 0, 0, 0), (0, 0, 0, 3)),
                                        ((8, 0, 16, 8), (3, 3, 3, 3)), ((2, 10, 2, 18), (0, 0, 0, 0)), ((3, 3, 11, 3), (5, 5, 5, 5))])
def test_strides(cuda_ok, n, more, start, dtype):
    Case(23, n, dtype, LAYER, RMS, more=more, start=start).check_backward()


@pytest.mark.parametrize("rows", [1, 2, 8, 30, 151, 152, 153, 1000, 5001])
def test_rows(cuda_ok, rows):
    Case(rows, 128, "bf16", RMS, LAYER).check_backward()
    Case(rows, 1031, "f32", RMS, RMS).check_backward()


@pytest.mark.parametrize("rows,n", [(70, 300), (9, 5000), (5, 9001), (3, 20000)])
def test_inside_a_partition(cuda_ok, rows, n):
    """A quarter of the SMs, where long rows are read several times instead of being
    shared by clusters."""
    part = G.goldy_partition_create(32, 1)
    _, (stream,) = G.goldy_partition_query(part, 1)
    for dtype in ("bf16", "f32"):
        c = Case(rows, n, dtype, LAYER, RMS)
        c.stream = stream
        torch.cuda.synchronize()
        c.check_backward()


def test_many_rows(cuda_ok):
    Case(70000, 40, "bf16", RMS, RMS).check_backward()
    Case(30001, 37, "bf16", RMS, LAYER).check_backward()
    Case(5003, 1023, "bf16", LAYER, RMS).check_backward()
    Case(5003, 517, "f32", LAYER, RMS).check_backward()


@pytest.mark.parametrize("n", [120, 5000])
def test_some_gradients(cuda_ok, n):
    """Those that are asked for, added to what is there."""
    whole = Case(30, n, "f32", LAYER, LAYER).check_backward()[-1]
    for wanted in ([], ["gate"], ["beta_f"], ["gamma_y", "gamma_f"]):
        got = Case(30, n, "f32", LAYER, LAYER).check_backward(wanted=wanted)[-1]
        assert all(torch.equal(got[k], whole[k]) for k in wanted)
    Case(30, n, "f32", LAYER, LAYER).check_backward(accumulate=True)


def test_far_apart(cuda_ok):
    """Rows more than 2^32 bytes, and elements, apart from the first: 70000 rows of a
    stride of 70000."""
    rows, n, ld = 70000, 16, 70000
    make = lambda fill=None: Rows(rows, n, torch.bfloat16, ld, 0, fill)  # noqa: E731
    gen = gen_of(1)
    x, f = (make(torch.randn(rows, n, generator=gen, device="cuda")) for _ in range(2))
    s, y, near = make(), make(), Case(rows, n, "bf16", LAYER, RMS)
    d = G.residual_norm_desc(rows, n, LAYER, RMS, alpha=0.75, ldx=ld, ldf=ld, lds=ld, ldy=ld)
    near.x.t.copy_(x.t)
    near.f.t.copy_(f.t)
    s2, y2, stats = near.check_forward()
    G.goldy_residual_norm_forward(d, near.params, x.ptr, f.ptr, s.ptr, y.ptr)
    torch.cuda.synchronize()
    assert torch.equal(s.t, s2.t) and torch.equal(y.t, y2.t)
    dx, df, dx2, df2 = make(), make(), near.new(0), near.new(1)
    near.backward(y2, s2, s2, stats, dx2, df2, wanted=[])
    G.goldy_residual_norm_backward(d, near.params, y.ptr, s.ptr, f.ptr, s.ptr, stats.data_ptr(), dx.ptr, df.ptr)
    torch.cuda.synchronize()
    assert torch.equal(dx.t, dx2.t) and torch.equal(df.t, df2.t)


def test_no_rows(cuda_ok):
    c = Case(0, 50, "f32", RMS, RMS)
    rows = [c.new(0) for _ in range(5)]
    for accumulate, want in ((False, 0.0), (True, 3.0)):
        grads = c.backward(rows[0], rows[1], rows[2], torch.zeros(4, 1, device="cuda"), rows[3], rows[4], accumulate=accumulate)
        assert all((g == want).all() for g in grads.values())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [100, 1001, 6000, 9001, 33000, 66001])
def test_in_place(cuda_ok, n, dtype):
    """Results over inputs give the same bits."""
    make = lambda: Case(25, n, dtype, RMS, LAYER)  # noqa: E731
    s, y, stats = make().check_forward()
    for s_is, y_is in (("x", "f"), ("f", "x"), ("x", None), (None, "x")):
        c = make()
        s2, y2 = getattr(c, s_is) if s_is else c.new(2), getattr(c, y_is) if y_is else c.new(3)
        G.goldy_residual_norm_forward(c.d, c.params, c.x.ptr, c.f.ptr, s2.ptr, y2.ptr)
        torch.cuda.synchronize()
        assert torch.equal(s2.t, s.t) and torch.equal(y2.t, y.t)
    dy, ds, s, stats, dx, df, grads = make().check_backward()
    for dx_is, df_is in ((1, 2), (0, 1), (2, 0), (3, 2), (1, 3)):
        c = make()
        arrays = [c.new(3, dy.t), c.new(2, ds.t), c.f, c.new(2, s.t)]
        got = c.backward(arrays[0], arrays[1], arrays[3], stats, arrays[dx_is], arrays[df_is])
        assert torch.equal(arrays[dx_is].t, dx.t) and torch.equal(arrays[df_is].t, df.t)
        assert all(torch.equal(got[k], grads[k]) for k in grads)


@pytest.mark.parametrize("n", [256, 1000, 5000])
def test_rows_far_from_zero(cuda_ok, n):
    """A mean of 1000 deviations: the bound has it through the sizes of the terms."""
    Case(40, n, "f32", LAYER, LAYER, far=1000.0).check_backward()


@pytest.mark.parametrize("norm_f", [NONE, LAYER, RMS])
@pytest.mark.parametrize("norm_y", [NONE, LAYER, RMS])
def test_automatic_differentiation(cuda_ok, norm_f, norm_y):
    """fp32 gradients against those of the fp64 forward pass.  S and the statistics
    are rounded to fp32 between the two, which the bound's margin (steps * u, three
    times here) covers."""
    c = Case(19, 200, "f32", norm_f, norm_y)
    dy, ds, s, stats, dx, df, grads = c.check_backward()
    for k in NAMES:
        c.v[k] = c.v[k].clone().requires_grad_(True)
    x, f = c.x.t.double().requires_grad_(True), c.f.t.double().requires_grad_(True)
    rs, _, ry, _, _ = c.forward64(x, f)
    loss = (rs * ds.t.double()).sum() + ((ry * dy.t.double()).sum() if norm_y else 0.0)
    loss.backward()
    with torch.no_grad():
        for k in NAMES:
            c.v[k] = c.v[k].detach()
        sizes = c.gradients64(dy.t.double(), ds.t.double(), c.f.t.double(), s.t.double(), stats)
        k3 = 3 * (steps(c.n) + 200) * U
        within(dx.t, x.grad, k3 * sizes[0][1], "dX")
        within(df.t, f.grad, k3 * sizes[1][1], "dF")
    grads64 = dict(zip(NAMES, torch.autograd.grad(_loss(c, dy, ds), [c.v[k] for k in NAMES], allow_unused=True)))
    for k, g in grads.items():
        within(g, grads64[k], k3 * sizes[2][k][1], "d" + k)


def _loss(c, dy, ds):
    for k in NAMES:
        c.v[k] = c.v[k].clone().requires_grad_(True)
    s, _, y, _, _ = c.forward64(c.x.t.double(), c.f.t.double())
    return (s * ds.t.double()).sum() + ((y * dy.t.double()).sum() if c.norm_y else 0.0)


def test_differences(cuda_ok):
    """dX and dF against central differences of the fp64 forward pass along random
    directions: with a step of 1e-5 their error is 1e-10 of the curvature and 1e-11
    of the loss, far below fp32's."""
    c = Case(6, 90, "f32", RMS, LAYER)
    dy, ds, s, stats, dx, df, grads = c.check_backward()
    gen = gen_of(12)
    x, f = c.x.t.double(), c.f.t.double()

    def loss(x, f):
        s, _, y, _, _ = c.forward64(x, f)
        return float((s * ds.t.double()).sum() + (y * dy.t.double()).sum())

    sizes = c.gradients64(dy.t.double(), ds.t.double(), f, s.t.double(), stats)
    for _ in range(5):
        a, b = (torch.randn(6, 90, generator=gen, device="cuda").double() for _ in range(2))
        h = 1e-5
        slope = (loss(x + h * a, f + h * b) - loss(x - h * a, f - h * b)) / (2 * h)
        got = float((dx.t.double() * a).sum() + (df.t.double() * b).sum())
        size = float((sizes[0][1] * a.abs()).sum() + (sizes[1][1] * b.abs()).sum())
        assert abs(got - slope) <= 3 * steps(c.n) * U * size + 1e-6 * abs(slope)
