"""Argument checks of the router, of tokens sorted by expert, of the residual
norms and of the 8-bit rows: refused before any CUDA call, so they run without a
GPU."""
import pytest

from paper_2409_02227_gb300 import goldy as G
from test_layers_abi import A, BAD, changed, refused

ROOM = 1 << 40


@pytest.mark.parametrize("fields", [dict(rows=-1), dict(rows=1 << 41), dict(experts=0), dict(experts=G.GOLDY_MAX_GROUPS + 1),
                                    dict(k=0), dict(k=65), dict(k=33, experts=64), dict(ld=63), dict(ldd=10),
                                    dict(ld=1 << 60), dict(over=2), dict(over=-1), dict(scale=float("inf")),
                                    dict(scale=float("nan")), dict(reserved=1)])
def test_router_descriptor(fields):
    d = lambda: changed(G.router_desc(32, 64, 8), **fields)  # noqa: E731
    refused(BAD, G.goldy_router_forward, d(), A, A, A)
    refused(BAD, G.goldy_router_backward, d(), A, A, A, A)


def test_router_pointers():
    d = G.router_desc(32, 64, 8)
    refused(G.GOLDY_ERR_UNSUPPORTED, G.goldy_router_forward, changed(G.router_desc(32, 64, 8), dtype=2), A, A, A)
    for at in range(3):
        for wrong in (0, A + 2):
            refused(BAD, G.goldy_router_forward, d, *[wrong if i == at else A for i in range(3)])
    for at in range(4):
        for wrong in (0, A + 2):
            refused(BAD, G.goldy_router_backward, d, *[wrong if i == at else A for i in range(4)])
    refused(BAD, G.goldy_router_backward, G.router_desc(32, 64, 8, ldd=70), A, A, A, A)          # in place, another stride
    refused(BAD, G.goldy_router_forward, G.router_desc(32, 64, 8, dtype=G.GOLDY_BF16), A + 1, A, A)
    G.goldy_router_forward(G.router_desc(0, 64, 8), 0, 0, 0)
    G.goldy_router_backward(G.router_desc(0, 64, 8), 0, 0, 0, 0)


@pytest.mark.parametrize("fields", [dict(rows=-1), dict(rows=1 << 31), dict(rows=1 << 30), dict(k=0), dict(k=33),
                                    dict(groups=0), dict(groups=G.GOLDY_MAX_GROUPS + 1), dict(width=-1), dict(ldx=99),
                                    dict(lde=99), dict(ldr=99), dict(lde=1 << 58), dict(reserved=1)])
def test_route_descriptor(fields):
    d = lambda: changed(G.route_desc(32, 2, 8, 100), **fields)  # noqa: E731
    refused(BAD, G.goldy_route_query, d())
    refused(BAD, G.goldy_route_sort, d(), A, A, A, workspace=A, workspace_bytes=ROOM)
    refused(BAD, G.goldy_route_dispatch, d(), A, A, A)
    refused(BAD, G.goldy_route_combine, d(), A, A, A)
    refused(BAD, G.goldy_route_combine_grad, d(), A, A, A, A, A, A)


def test_route_pointers():
    d = G.route_desc(32, 2, 8, 100, dtype=G.GOLDY_F32)
    refused(G.GOLDY_ERR_UNSUPPORTED, G.goldy_route_query, changed(G.route_desc(32, 2, 8, 100), dtype=2))
    for wrong in (0, A + 2):
        for at in range(3):
            args = [wrong if i == at else A for i in range(3)]
            refused(BAD, G.goldy_route_sort, d, *args)
            refused(BAD, G.goldy_route_dispatch, d, *args)
            refused(BAD, G.goldy_route_combine, d, *args)
        for at in (0, 1, 2, 4):
            refused(BAD, G.goldy_route_combine_grad, d, *[wrong if i == at else A for i in range(6)])
    refused(BAD, G.goldy_route_sort, d, A, A, A, source=A + 2)
    refused(BAD, G.goldy_route_combine, d, A, A, A, weights=A + 2)
    refused(BAD, G.goldy_route_combine, d, A, A, A, residual=A + 1)
    refused(BAD, G.goldy_route_combine, G.route_desc(32, 2, 8, 100, ldr=104), A, A, A + 4096, residual=A + 4096)
    refused(BAD, G.goldy_route_combine_grad, d, A, A, A, A + 2, A, A)
    refused(BAD, G.goldy_route_combine_grad, d, A, A, A, A, A, A + 2)
    big = G.route_desc(1 << 16, 4, 64)
    need = G.goldy_route_query(big)
    assert need > 65536
    refused(BAD, G.goldy_route_sort, big, A, A, A)
    refused(BAD, G.goldy_route_sort, big, A, A, A, workspace=A + 128, workspace_bytes=ROOM)
    refused(G.GOLDY_ERR_NOMEM, G.goldy_route_sort, big, A, A, A, workspace=A, workspace_bytes=need - 1)
    for empty in (G.route_desc(0, 2, 8, 100), G.route_desc(32, 2, 8, 0)):
        G.goldy_route_dispatch(empty, 0, 0, 0)
        G.goldy_route_combine(empty, 0, 0, 0)
        G.goldy_route_combine_grad(empty, 0, 0, 0, 0, 0)


RMS, LAYER, NONE = G.GOLDY_NORM_RMS, G.GOLDY_NORM_LAYER, G.GOLDY_NORM_NONE


@pytest.mark.parametrize("fields", [dict(rows=-1), dict(n=-1), dict(n=(1 << 30) + 1), dict(ldx=99), dict(ldf=99), dict(lds=99),
                                    dict(ldy=99), dict(lds=1 << 59), dict(norm_f=3), dict(norm_y=-1), dict(eps=-1.0),
                                    dict(eps=float("nan")), dict(alpha=float("inf")), dict(alpha=float("nan")),
                                    dict(reserved=1)])
def test_residual_norm_descriptor(fields):
    d = lambda: changed(G.residual_norm_desc(32, 100), **fields)  # noqa: E731
    refused(BAD, G.goldy_residual_norm_query, d())
    refused(BAD, G.goldy_residual_norm_forward, d(), None, A, A, A, 2 * A)
    refused(BAD, G.goldy_residual_norm_backward, d(), None, A, A, A, A, A, 2 * A, 3 * A)


def test_residual_norm_pointers():
    for field in ("dtype", "param_dtype"):
        refused(G.GOLDY_ERR_UNSUPPORTED, G.goldy_residual_norm_query, changed(G.residual_norm_desc(4, 100), **{field: 2}))
    d, none = G.residual_norm_desc(32, 100, dtype=G.GOLDY_F32), G.residual_norm_desc(32, 100, NONE, NONE)
    for wrong in (0, A + 2):
        for at in range(4):                                          # X, F, S, Y
            refused(BAD, G.goldy_residual_norm_forward, d, None, *[wrong if i == at else (i + 1) * A for i in range(4)])
        for at in (0, 2, 3, 4, 5, 6):                                # dY, F, S, stats, dX, dF
            refused(BAD, G.goldy_residual_norm_backward, d, None, *[wrong if i == at else (i + 1) * A for i in range(7)])
    refused(BAD, G.goldy_residual_norm_backward, d, None, A, A + 2, A, A, A, 2 * A, 3 * A)
    refused(BAD, G.goldy_residual_norm_forward, d, None, A, A, 2 * A, 3 * A, stats=A + 2)
    refused(BAD, G.goldy_residual_norm_forward, none, None, A, A, 2 * A, 3 * A)                     # Y without a norm
    refused(BAD, G.goldy_residual_norm_backward, none, None, A, A, A, A, A, 2 * A, 3 * A)           # dY without a norm
    refused(BAD, G.goldy_residual_norm_backward, none, None, 0, 0, A, A, A, 2 * A, 3 * A)           # no gradient at all
    refused(BAD, G.goldy_residual_norm_forward, d, None, A, A, 2 * A, 2 * A)                        # S is Y
    refused(BAD, G.goldy_residual_norm_backward, d, None, A, A, A, A, A, 2 * A, 2 * A)              # dX is dF
    wide = lambda **ld: G.residual_norm_desc(32, 100, **ld)  # noqa: E731
    refused(BAD, G.goldy_residual_norm_forward, wide(lds=104), None, A, 2 * A, A, 3 * A)
    refused(BAD, G.goldy_residual_norm_forward, wide(ldf=104), None, A, 2 * A, 2 * A, 3 * A)
    refused(BAD, G.goldy_residual_norm_forward, wide(ldx=104), None, A, 2 * A, 3 * A, A)
    refused(BAD, G.goldy_residual_norm_backward, wide(ldx=104), None, A, 2 * A, 3 * A, 4 * A, 5 * A, 2 * A, 6 * A)
    refused(BAD, G.goldy_residual_norm_backward, wide(ldf=104), None, A, 2 * A, 3 * A, 4 * A, 5 * A, 6 * A, A)
    for name in ("gate", "gamma_f", "beta_f", "gamma_y", "beta_y"):
        p = G.residual_norm_params(**{name: A + 2})
        refused(BAD, G.goldy_residual_norm_forward, d, p, A, 2 * A, 3 * A, 4 * A)
        refused(BAD, G.goldy_residual_norm_backward, d, None, A, A, A, A, A, 2 * A, 3 * A, p, A, ROOM)
        if name != "gate":
            p = G.residual_norm_params(**{name: A})
            refused(BAD, G.goldy_residual_norm_forward, none, p, A, 2 * A, 3 * A)
            refused(BAD, G.goldy_residual_norm_backward, none, None, 0, A, A, A, A, 2 * A, 3 * A, p, A, ROOM)
    want, need = G.residual_norm_params(gate=A), G.goldy_residual_norm_query(d)
    refused(BAD, G.goldy_residual_norm_backward, d, None, A, A, A, A, A, 2 * A, 3 * A, want)
    refused(G.GOLDY_ERR_NOMEM, G.goldy_residual_norm_backward, d, None, A, A, A, A, A, 2 * A, 3 * A, want, A, need - 1)
    G.goldy_residual_norm_forward(G.residual_norm_desc(0, 100), None, 0, 0, 0)
    G.goldy_residual_norm_forward(G.residual_norm_desc(32, 0), None, 0, 0, 0)
    G.goldy_residual_norm_backward(G.residual_norm_desc(0, 100), None, 0, 0, 0, 0, 0, 0, 0)
    assert G.goldy_residual_norm_query(G.residual_norm_desc(32, 0)) == 0


def test_keep8():
    for fields in (dict(rows=-1), dict(n=-1), dict(n=(1 << 30) + 1), dict(ldz=99), dict(ldh=99), dict(ldz=1 << 59), dict(act=5),
                   dict(act=-1), dict(reserved=1)):
        d = changed(G.keep8_desc(32, 100), **fields)
        refused(BAD, G.goldy_keep8_query, d)
        refused(BAD, G.goldy_keep8_pack, d, A, A, A)
        refused(BAD, G.goldy_keep8_unpack, d, A, A, A)
    refused(G.GOLDY_ERR_UNSUPPORTED, G.goldy_keep8_query, changed(G.keep8_desc(32, 100), dtype=2))
    d = G.keep8_desc(32, 100)
    assert G.goldy_keep8_query(d) == (32 * 4 * 32, 32 * 4)
    assert G.goldy_keep8_query(G.keep8_desc(0, 100)) == (0, 0)
    for at in range(3):
        refused(BAD, G.goldy_keep8_pack, d, *[0 if i == at else A for i in range(3)])
    refused(BAD, G.goldy_keep8_pack, d, A + 1, A, A)
    refused(BAD, G.goldy_keep8_pack, d, A, A + 8, A)
    refused(BAD, G.goldy_keep8_unpack, d, 0, A, A)
    refused(BAD, G.goldy_keep8_unpack, d, A, 0, A)
    refused(BAD, G.goldy_keep8_unpack, d, A, A)
    refused(BAD, G.goldy_keep8_unpack, d, A + 8, A, A)
    refused(BAD, G.goldy_keep8_unpack, d, A, A, A + 1)
    refused(BAD, G.goldy_keep8_unpack, d, A, A, 0, A + 1)
    refused(BAD, G.goldy_keep8_unpack, d, A, A, A, A)
    for empty in (G.keep8_desc(0, 100), G.keep8_desc(32, 0)):
        G.goldy_keep8_pack(empty, 0, 0, 0)
        G.goldy_keep8_unpack(empty, 0, 0)
