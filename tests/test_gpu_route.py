"""Tokens sorted by expert and back, against plain indexing.

Bounds.  A sum of k weighted rows and R has k + 1 steps of fp32, so (k + 2) u of the
sum of the terms' sizes, then one rounding to the result's type; a product is
rounded to fp32 and to the type; a dot product over `width` elements has at most
width / 8 + 40 steps (a warp's lanes take blocks of 4 or 8, each added up in
order), so that many u of the sum of the products' sizes."""
import pytest
import torch

from expert_ops_util import GUARD, HALF, TYPES, U, Rows, gen_of, within, workspace
from paper_2409_02227_gb300 import goldy as G

pytestmark = pytest.mark.gpu


def sort(d, ids, source=True):
    slots = ids.numel()
    offsets = torch.full((d.groups + 1,), -7, dtype=torch.int32, device="cuda")
    place = torch.full((slots,), -7, dtype=torch.int32, device="cuda")
    src = torch.full((slots,), -7, dtype=torch.int32, device="cuda")
    need = G.goldy_route_query(d)
    ws = workspace(need)
    G.goldy_route_sort(d, ids.data_ptr(), offsets.data_ptr(), place.data_ptr(), src.data_ptr() if source else 0,
                       ws.data_ptr() if need else 0, need)
    torch.cuda.synchronize()
    assert need == 0 or not ws[:65536].any()
    return offsets, place, src


def sorted_plainly(ids, groups):
    key = ids.flatten().long().cpu()
    key = torch.where((key < 0) | (key >= groups), groups, key)
    by, order = key.sort(stable=True)
    place = torch.empty_like(order)
    place[order] = torch.arange(len(order))
    offsets = torch.searchsorted(by, torch.arange(groups + 1))
    return offsets.int(), torch.where(key == groups, -1, place).int(), torch.where(by == groups, -1, order).int()


def check_sort(ids, rows, k, groups):
    offsets, place, src = sort(G.route_desc(rows, k, groups), ids)
    for got, want in zip((offsets, place, src), sorted_plainly(ids, groups)):
        assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("rows,k,groups", [(1, 1, 1), (1, 8, 64), (5, 3, 7), (16, 6, 64), (100, 2, 8), (511, 8, 31), (512, 8, 16),
                                           (513, 8, 16), (1024, 2, 16), (683, 3, 5), (4096, 1, 256), (4097, 1, 256), (1366, 3, 60), (3000, 32, 128),
                                           (700, 6, 2000), (1000, 5, 4096), (2, 1, 4096), (160001, 4, 33)])
def test_sort(cuda_ok, rows, k, groups):
    ids = torch.randint(-1, groups + 1, (rows, k), generator=gen_of(rows), device="cuda").int()
    check_sort(ids, rows, k, groups)


@pytest.mark.parametrize("rows", [1, 700, 5000, 20000])
def test_sort_of_strange_ids(cuda_ok, rows):
    """All slots of one expert, none of any, ids far out of range, one expert at the end."""
    for ids in (3, -1, 9, 1 << 30, -(1 << 31)):
        check_sort(torch.full((rows, 2), ids, dtype=torch.int32, device="cuda"), rows, 2, 9)
    ids = torch.full((rows, 2), -5, dtype=torch.int32, device="cuda")
    ids[-1, -1] = 8
    check_sort(ids, rows, 2, 9)


def test_sort_without_slots(cuda_ok):
    offsets, _, _ = sort(G.route_desc(0, 2, 70), torch.empty(0, 2, dtype=torch.int32, device="cuda"))
    assert (offsets == 0).all()


def test_sort_without_source(cuda_ok):
    for rows in (10, 9000):
        ids = torch.randint(-1, 8, (rows, 2), generator=gen_of(rows), device="cuda").int()
        with_, without = sort(G.route_desc(rows, 2, 8), ids), sort(G.route_desc(rows, 2, 8), ids, False)
        assert torch.equal(with_[0], without[0]) and torch.equal(with_[1], without[1]) and (without[2] == -7).all()


def test_sort_again_in_one_workspace(cuda_ok):
    """A workspace that other sizes have used."""
    ws = workspace(max(G.goldy_route_query(G.route_desc(9000, 2, g)) for g in (4, 500)))
    for seed, groups in enumerate((500, 4, 500, 70)):
        ids = torch.randint(-1, groups + 1, (9000, 2), generator=gen_of(seed), device="cuda").int()
        place = torch.empty(18000, dtype=torch.int32, device="cuda")
        offsets = torch.empty(groups + 1, dtype=torch.int32, device="cuda")
        G.goldy_route_sort(G.route_desc(9000, 2, groups), ids.data_ptr(), offsets.data_ptr(), place.data_ptr(), 0, ws.data_ptr(),
                           ws.numel())
        want = sorted_plainly(ids, groups)
        assert torch.equal(offsets.cpu(), want[0]) and torch.equal(place.cpu(), want[1])


# ---- rows ------------------------------------------------------------------------

SHAPES = [  # rows, k, groups, width, strides behind the width (tokens, experts, R), elements to start on
    (1, 1, 1, 1, (0, 0, 0), (0, 0, 0)), (3, 2, 4, 7, (0, 0, 0), (0, 0, 0)), (40, 3, 5, 8, (0, 0, 0), (0, 0, 0)),
    (40, 3, 5, 9, (1, 2, 3), (1, 2, 3)), (33, 9, 12, 64, (0, 0, 0), (0, 0, 0)), (33, 9, 12, 64, (8, 0, 16), (0, 8, 0)),
    (33, 9, 12, 64, (0, 0, 0), (1, 0, 0)), (33, 9, 12, 64, (0, 0, 0), (0, 3, 0)), (33, 9, 12, 64, (0, 0, 0), (0, 0, 5)),
    (20, 32, 40, 100, (1, 0, 4), (0, 0, 0)), (50, 2, 6, 1111, (0, 0, 0), (0, 0, 0)), (50, 2, 6, 1111, (5, 3, 7), (7, 6, 1)),
    (200, 6, 64, 2048, (0, 0, 0), (0, 0, 0)), (9, 4, 4, 8200, (0, 0, 0), (0, 0, 0)), (9, 4, 4, 8193, (2, 0, 1), (4, 0, 2)),
    (3000, 1, 16, 72, (0, 0, 0), (0, 0, 0)),
]


class Case:
    def __init__(self, dtype, rows, k, groups, width, more, start, lost=0.1):
        gen, t = gen_of(rows + width), TYPES[dtype][0]
        self.dtype, self.rows, self.k, self.width = t, rows, k, width
        self.ids = torch.randint(0, groups, (rows, k), generator=gen, device="cuda").int()
        self.ids[torch.rand(rows, k, generator=gen, device="cuda") < lost] = -1
        if rows > 2:
            self.ids[1] = -1                                # a token without any expert
        rnd = lambda n: torch.randn(n, width, generator=gen, device="cuda")  # noqa: E731
        self.lds, self.start = [width + m for m in more], start
        self.x, self.r = Rows(rows, width, t, self.lds[0], start[0], rnd(rows)), Rows(rows, width, t, self.lds[2], start[2], rnd(rows))
        self.e = Rows(rows * k, width, t, self.lds[1], start[1], rnd(rows * k))
        self.weights = torch.randn(rows, k, generator=gen, device="cuda")
        self.d = G.route_desc(rows, k, groups, width, dtype=TYPES[dtype][1], ldx=self.lds[0], lde=self.lds[1], ldr=self.lds[2])
        self.offsets, self.place, _ = sort(self.d, self.ids)
        self.at = self.place.view(rows, k).long()
        behind = int(self.offsets[-1])
        self.e.t[behind:] = float("nan")                    # rows behind the last are never read
        self.all_e = self.e.t[self.at.clamp(min=0)].double()
        self.all_e[self.at < 0] = 0.0

    def token_rows(self):
        return Rows(self.rows, self.width, self.dtype, self.lds[0], self.start[0])

    def expert_rows(self):
        return Rows(self.rows * self.k, self.width, self.dtype, self.lds[1], self.start[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_dispatch(cuda_ok, shape, dtype):
    c, e = Case(dtype, *shape), None
    e = c.expert_rows()
    G.goldy_route_dispatch(c.d, c.x.ptr, c.place.data_ptr(), e.ptr)
    torch.cuda.synchronize()
    want = torch.full_like(e.t, GUARD)                      # rows without a slot stay as they were
    there = c.at.flatten() >= 0
    want[c.at.flatten()[there]] = c.x.t.repeat_interleave(c.k, 0)[there]
    assert torch.equal(e.t, want) and e.guarded() and c.x.guarded()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("weighted,residual", [(True, True), (True, False), (False, True), (False, False)])
def test_combine(cuda_ok, shape, dtype, weighted, residual):
    c = Case(dtype, *shape)
    y = c.token_rows()
    G.goldy_route_combine(c.d, c.e.ptr, c.place.data_ptr(), y.ptr, c.weights.data_ptr() if weighted else 0,
                          c.r.ptr if residual else 0)
    torch.cuda.synchronize()
    terms = c.all_e * (c.weights.double()[:, :, None] if weighted else 1.0)
    ref, size = terms.sum(1), terms.abs().sum(1)
    if residual:
        ref, size = ref + c.r.t.double(), size + c.r.t.double().abs()
    within(y.t, ref, HALF[c.dtype] * ref.abs() + (c.k + 2) * U * size, "y")
    assert y.guarded()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_combine_grad(cuda_ok, shape, dtype):
    c = Case(dtype, *shape)
    dy = c.x
    de, dw = c.expert_rows(), torch.full((c.rows, c.k), float("nan"), device="cuda")
    G.goldy_route_combine_grad(c.d, dy.ptr, c.e.ptr, c.place.data_ptr(), c.weights.data_ptr(), de.ptr, dw.data_ptr())
    torch.cuda.synchronize()
    products = c.all_e * dy.t.double()[:, None]
    within(dw, products.sum(2), (c.width / 8 + 40) * U * products.abs().sum(2), "dweights")
    there = c.at.flatten() >= 0
    want = torch.full(de.t.shape, GUARD, dtype=torch.float64, device="cuda")
    want[c.at.flatten()[there]] = (c.weights.double()[:, :, None] * dy.t.double()[:, None]).view(-1, c.width)[there]
    tol = (HALF[c.dtype] + U) * want.abs() * 1.01
    tol[int(c.offsets[-1]):] = 0.0
    within(de.t, want, tol, "dE")
    assert de.guarded()
    # without the dot products, without weights, and over E itself
    alone = c.expert_rows()
    G.goldy_route_combine_grad(c.d, dy.ptr, 0, c.place.data_ptr(), c.weights.data_ptr(), alone.ptr)
    ones, copied = c.expert_rows(), c.expert_rows()
    G.goldy_route_combine_grad(c.d, dy.ptr, 0, c.place.data_ptr(), 0, ones.ptr)
    G.goldy_route_dispatch(c.d, dy.ptr, c.place.data_ptr(), copied.ptr)
    again = torch.empty_like(dw)
    G.goldy_route_combine_grad(c.d, dy.ptr, c.e.ptr, c.place.data_ptr(), c.weights.data_ptr(), c.e.ptr, again.data_ptr())
    torch.cuda.synchronize()
    assert torch.equal(alone.t, de.t) and torch.equal(ones.t, copied.t) and torch.equal(again, dw)
    behind = int(c.offsets[-1])
    assert torch.equal(c.e.t[:behind], de.t[:behind]) and torch.isnan(c.e.t[behind:]).all()


def test_combine_over_the_residual(cuda_ok):
    for shape in (SHAPES[4], SHAPES[6], SHAPES[11]):
        c = Case("bf16", *shape)
        d = G.route_desc(c.rows, c.k, 99, c.width, ldx=c.lds[2], lde=c.lds[1], ldr=c.lds[2])
        y = Rows(c.rows, c.width, c.dtype, c.lds[2], c.start[2])
        G.goldy_route_combine(d, c.e.ptr, c.place.data_ptr(), y.ptr, c.weights.data_ptr(), c.r.ptr)
        G.goldy_route_combine(d, c.e.ptr, c.place.data_ptr(), c.r.ptr, c.weights.data_ptr(), c.r.ptr)
        torch.cuda.synchronize()
        assert torch.equal(y.t, c.r.t) and c.r.guarded()


def test_dispatch_gradient_is_combine(cuda_ok):
    """<dispatch(x), g> = <x, combine(g)> in integers, where nothing rounds."""
    c = Case("f32", 50, 4, 6, 40, (0, 0, 0), (0, 0, 0))
    x = torch.randint(-8, 9, (50, 40), generator=gen_of(1), device="cuda").float()
    g = torch.randint(-8, 9, (200, 40), generator=gen_of(2), device="cuda").float()
    e, dx = torch.zeros(200, 40, device="cuda"), torch.empty(50, 40, device="cuda")
    G.goldy_route_dispatch(c.d, x.data_ptr(), c.place.data_ptr(), e.data_ptr())
    G.goldy_route_combine(c.d, g.data_ptr(), c.place.data_ptr(), dx.data_ptr())
    torch.cuda.synchronize()
    assert float((e * g).sum()) == float((x * dx).sum())


def test_far_apart(cuda_ok):
    """Experts' rows more than 2^32 elements apart."""
    rows, k, width, lde = 40000, 2, 24, 60000
    d = G.route_desc(rows, k, 8, width, lde=lde)
    ids = torch.randint(0, 8, (rows, k), generator=gen_of(1), device="cuda").int()
    offsets, place, _ = sort(d, ids)
    x = torch.randn(rows, width, generator=gen_of(2), device="cuda").bfloat16()
    e = torch.zeros(rows * k, lde, dtype=torch.bfloat16, device="cuda")
    G.goldy_route_dispatch(d, x.data_ptr(), place.data_ptr(), e.data_ptr())
    y, dw = torch.empty_like(x), torch.empty(rows, k, device="cuda")
    G.goldy_route_combine(d, e.data_ptr(), place.data_ptr(), y.data_ptr())
    torch.cuda.synchronize()
    assert torch.equal(e[place.long(), :width], x.repeat_interleave(k, 0)) and torch.equal(y, 2 * x)
    G.goldy_route_combine_grad(d, x.data_ptr(), e.data_ptr(), place.data_ptr(), 0, e.data_ptr(), dw.data_ptr())
    torch.cuda.synchronize()
    assert torch.equal(dw[:, 0], dw[:, 1]) and torch.equal(e[place.long(), :width], x.repeat_interleave(k, 0))
    assert not e[:, width:].any()


def test_rows_without_elements(cuda_ok):
    """Only the weights' gradient has something to write: zeros."""
    d, place = G.route_desc(6, 2, 3, 0), torch.arange(12, dtype=torch.int32, device="cuda")
    dw = torch.full((12,), 5.0, device="cuda")
    odd = torch.zeros(8, dtype=torch.uint16, device="cuda").data_ptr() + 2
    G.goldy_route_combine_grad(d, odd, odd, place.data_ptr(), 0, odd, dw.data_ptr())
    torch.cuda.synchronize()
    assert (dw == 0).all()


def test_places_out_of_range(cuda_ok):
    """Places that no slot can have count as -1 and reach no memory."""
    d = G.route_desc(4, 2, 3, 16, dtype=G.GOLDY_F32)
    place = torch.tensor([0, 8, -2, 1 << 30, 3, -(1 << 31), 7, 100], dtype=torch.int32, device="cuda")
    x = torch.randn(4, 16, generator=gen_of(1), device="cuda")
    e, y, r = Rows(8, 16, torch.float32), Rows(4, 16, torch.float32), torch.randn(4, 16, generator=gen_of(2), device="cuda")
    G.goldy_route_dispatch(d, x.data_ptr(), place.data_ptr(), e.ptr)
    e2 = torch.randn(8, 16, generator=gen_of(3), device="cuda")
    G.goldy_route_combine(d, e2.data_ptr(), place.data_ptr(), y.ptr, residual=r.data_ptr())
    torch.cuda.synchronize()
    assert torch.equal(e.t[[0, 3, 7]], x[[0, 2, 3]]) and (e.t[[1, 2, 4, 5, 6]] == GUARD).all() and e.guarded()
    assert torch.equal(y.t, r + torch.stack([e2[0], torch.zeros_like(e2[0]), e2[3], e2[7]]))
