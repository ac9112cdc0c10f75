"""Workspace sizes of the linear layer's calls, and sizes that are refused; host
code only."""
import pytest

from paper_2409_02227_gb300 import goldy as G

LARGEST = (1 << 31) - 1024


@pytest.mark.parametrize("rows,k,n,kw", [
    (32, LARGEST, LARGEST - 2, dict(groups=4096, ldw=LARGEST - 1)),     # W's padded copy: 2^75 bytes
    (32, LARGEST, LARGEST, dict(groups=4096)),
    (32, 1 << 20, 1 << 20, dict(groups=4096, stride_w=1 << 60)),
    (LARGEST, LARGEST, 8, {}),
    (LARGEST, 8, LARGEST, {}),
    (LARGEST, 8, 8, dict(ldx=LARGEST)),
    (LARGEST, 8, 8, dict(ldz=LARGEST)),
])
def test_arrays_beyond_any_memory_are_refused(rows, k, n, kw):
    """Sizes that wrapped around when the workspace was computed."""
    with pytest.raises(G.GoldyError) as e:
        G.goldy_linear_query(G.linear_desc(rows, k, n, **kw))
    assert e.value.status == G.GOLDY_ERR_INVALID_ARG


def test_long_strides_of_few_rows_are_not():
    G.goldy_linear_query(G.linear_desc(5, 72, 72, ldx=LARGEST, ldy=LARGEST, ldz=LARGEST, ldr=LARGEST))
    G.goldy_linear_query(G.linear_desc(300, 8192, 8192, groups=512, stride_w=1 << 32))
    G.goldy_linear_query(G.linear_desc(1 << 24, 8192, 8192))
