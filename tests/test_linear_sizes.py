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


@pytest.mark.parametrize("groups", [0, 1, 8, 64, 4096])
@pytest.mark.parametrize("rows", [1, 37, 500, 100000])
@pytest.mark.parametrize("k,n", [(4096, 1024), (75, 130), (64, 8), (1001, 77)])
def test_workspace_holds_what_the_calls_keep_there(rows, k, n, groups):
    """64 KiB of counters and, one call at a time, the bias gradient's partial rows
    (a slice's or an expert's, one more than their number apart from each other) or
    padded copies of both operands whose rows are off 16 bytes."""
    pad = lambda cols: (cols + 7) // 8 * 8  # noqa: E731
    experts = max(1, groups)
    x, y, w = rows * pad(k) * 2, rows * pad(n) * 2, experts * k * pad(n) * 2
    assert G.goldy_linear_query(G.linear_desc(rows, k, n, groups=groups)) >= 65536 + (1 + experts) * n * 4
    packed = G.goldy_linear_query(G.linear_desc(rows, k, n, groups=groups, ldx=k, ldw=n, ldy=n))
    x, y, w = x if k % 8 else 0, y if n % 8 else 0, w if n % 8 else 0
    assert packed >= 65536 + max(x + w, y + w, x + y)
    if rows > 1 and groups > 1 and n % 8:
        apart = G.linear_desc(rows, k, n, groups=groups, ldw=pad(n), ldy=pad(n), ldx=pad(k), stride_w=k * pad(n) + 4)
        assert G.goldy_linear_query(apart) >= 65536 + w       # experts off 16 bytes from one another
