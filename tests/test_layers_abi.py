"""Argument checks of the layer operators: refused before any CUDA call, so
they run without a GPU."""
import pytest

from paper_2409_02227_gb300 import goldy as G

A = 1 << 20            # an aligned address; never read, every call below is refused


def refused(status, call, *args, **kw):
    with pytest.raises(G.GoldyError) as e:
        call(*args, **kw)
    assert e.value.status == status, e.value
    assert G.goldy_last_error()


BAD = G.GOLDY_ERR_INVALID_ARG


def changed(d, **fields):
    for k, v in fields.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("fields", [dict(rows=-1), {"in": -1}, dict(out=-5), dict(rows=1 << 31), dict(ldx=63), dict(ldw=127),
                                    dict(ldy=100), dict(ldz=-1), dict(ldr=-8), dict(groups=-1),
                                    dict(groups=G.GOLDY_MAX_GROUPS + 1), dict(groups=2, stride_w=8), dict(stride_w=-8), dict(lddx=63),
                                    dict(act=5), dict(act=-1), dict(act_x=9), dict(reserved=1)])
def test_linear_descriptor(fields):
    refused(BAD, G.goldy_linear_query, changed(G.linear_desc(32, 64, 128), **fields))
    refused(BAD, G.goldy_linear_forward, changed(G.linear_desc(32, 64, 128), **fields), A, A, A)


@pytest.mark.parametrize("field", ["y_dtype", "dx_dtype", "dw_dtype", "bias_dtype"])
def test_linear_types(field):
    refused(G.GOLDY_ERR_UNSUPPORTED, G.goldy_linear_query, changed(G.linear_desc(32, 64, 128), **{field: 2}))


def test_linear_pointers():
    d = G.linear_desc(32, 64, 128)
    refused(BAD, G.goldy_linear_forward, d, 0, A, A)
    refused(BAD, G.goldy_linear_forward, d, A, 0, A)
    refused(BAD, G.goldy_linear_forward, d, A, A, 0)
    refused(BAD, G.goldy_linear_forward, d, A + 8, A, A)
    refused(BAD, G.goldy_linear_forward, d, A, A + 2, A)
    refused(BAD, G.goldy_linear_forward, d, A, A, A + 1)
    refused(BAD, G.goldy_linear_forward, d, A, A, A, bias=A + 1)
    refused(BAD, G.goldy_linear_forward, d, A, A, A, residual=A + 1)
    refused(BAD, G.goldy_linear_forward, d, A, A, A, z=A + 1)
    refused(BAD, G.goldy_linear_forward, changed(G.linear_desc(32, 64, 128), ldz=100), A, A, A, z=A)
    refused(BAD, G.goldy_linear_forward, changed(G.linear_desc(32, 64, 128), ldr=100), A, A, A, residual=A)
    odd = G.linear_desc(32, 60, 128, ldx=60)                     # rows of X off 16 bytes: a copy, so a workspace
    assert G.goldy_linear_query(odd) >= 65536 + 32 * 64 * 2
    assert G.goldy_linear_query(G.linear_desc(32, 64, 126, ldw=126)) >= 65536 + 64 * 128 * 2
    refused(BAD, G.goldy_linear_forward, odd, A + 1, A, A)
    refused(BAD, G.goldy_linear_forward, G.linear_desc(32, 64, 128, groups=2), A, A, A)             # no offsets
    refused(BAD, G.goldy_linear_forward, G.linear_desc(32, 64, 128, groups=2), A, A, A, offsets=A + 2)
    refused(BAD, G.goldy_linear_forward, d, A, A, A, offsets=A)


def test_gradient_pointers():
    d = G.linear_desc(32, 64, 128)
    refused(BAD, G.goldy_linear_input_grad, d, 0, A, A)
    refused(BAD, G.goldy_linear_input_grad, d, A, A, 0)
    refused(BAD, G.goldy_linear_input_grad, d, A, A, A, z=A)                                        # no activation
    refused(BAD, G.goldy_linear_input_grad, G.linear_desc(32, 64, 128, act_x=G.GOLDY_ACT_GELU), A, A, A)
    refused(BAD, G.goldy_linear_weight_grad, d, 0, A, A)
    refused(BAD, G.goldy_linear_weight_grad, d, A, 0, A)
    refused(BAD, G.goldy_linear_weight_grad, d, A, A, 0)
    refused(BAD, G.goldy_linear_weight_grad, d, A, A, A + 2)                                        # fp32 result
    refused(BAD, G.goldy_linear_bias_grad, d, 0, A, workspace=A, workspace_bytes=1 << 30)
    refused(BAD, G.goldy_linear_bias_grad, d, A, 0, workspace=A, workspace_bytes=1 << 30)
    refused(BAD, G.goldy_linear_bias_grad, d, A, A, z=A, dz=A, workspace=A, workspace_bytes=1 << 30)
    act = G.linear_desc(32, 64, 128, act=G.GOLDY_ACT_SILU)
    refused(BAD, G.goldy_linear_bias_grad, act, A, A, z=A, workspace=A, workspace_bytes=1 << 30)
    refused(BAD, G.goldy_linear_bias_grad, d, A, A)                                                 # no workspace
    refused(G.GOLDY_ERR_NOMEM, G.goldy_linear_bias_grad, d, A, A, workspace=A, workspace_bytes=65536)


def test_layernorm():
    d = G.layernorm_desc(4, 100)
    for fields in (dict(rows=-1), dict(n=-1), dict(ldx=99), dict(ldy=99), dict(eps=-1.0), dict(eps=float("nan")),
                   dict(eps=float("inf")), dict(reserved=1)):
        refused(BAD, G.goldy_layernorm_query, changed(G.layernorm_desc(4, 100), **fields))
    for field in ("dtype", "param_dtype"):
        refused(G.GOLDY_ERR_UNSUPPORTED, G.goldy_layernorm_query, changed(G.layernorm_desc(4, 100), **{field: 3}))
    refused(BAD, G.goldy_layernorm_forward, d, 0, 0, 0, A)
    refused(BAD, G.goldy_layernorm_forward, d, A, 0, 0, 0)
    refused(BAD, G.goldy_layernorm_forward, d, A + 1, 0, 0, A)
    refused(BAD, G.goldy_layernorm_forward, d, A, A + 1, 0, A)
    refused(BAD, G.goldy_layernorm_forward, d, A, 0, 0, A, A + 2)
    refused(BAD, G.goldy_layernorm_backward, d, A, A, 0, 0, A, A)                                   # no mean
    refused(BAD, G.goldy_layernorm_backward, d, A, 0, 0, A, A, A)
    refused(BAD, G.goldy_layernorm_backward, d, A, A, 0, A, A, A, A, A)                             # no workspace
    refused(G.GOLDY_ERR_NOMEM, G.goldy_layernorm_backward, d, A, A, 0, A, A, A, A, A, A, 1000)


def test_nothing_to_do():
    G.goldy_linear_forward(G.linear_desc(0, 64, 128), 0, 0, 0)
    G.goldy_linear_input_grad(G.linear_desc(32, 0, 128), 0, 0, 0)
    G.goldy_linear_weight_grad(G.linear_desc(32, 64, 0), 0, 0, 0)
    G.goldy_layernorm_forward(G.layernorm_desc(0, 64), 0, 0, 0, 0)
    assert G.goldy_layernorm_query(G.layernorm_desc(4, 0)) == 0


def test_workspace_covers_every_group_size():
    """The query's bound grows with the groups and holds for a single row."""
    for rows in (1, 37, 500):
        for groups in (0, 1, 8, 64):
            assert G.goldy_linear_query(G.linear_desc(rows, 4096, 1024, groups=groups)) >= 0
