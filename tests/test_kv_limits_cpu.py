"""Sizes that the C ABI of the key/value cache refuses because no launch takes
them.  Pointers are never dereferenced: every call here is refused on the host."""

import pytest

from test_kv_cpu import EUNSUPPORTED, FAKE, L, OK, append, batch, cache, read  # noqa: F401  (L: a fixture)

WORKGROUP = 128
MOST = 1 << 32     # threads of a launch: fewer than this


def one_head(D):
    return cache(kv_heads=1, head_dim=D, pages=8)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [(1 << 25), (1 << 25) - 1])
def test_launches_of_2_to_the_32_threads_are_refused(L, rows, D):  # noqa: F811
    """A row takes a workgroup however few its heads are.  One key/value head and no query: 2^25 rows times two heads
    are within the bound on rows times heads, and their workgroups 2^32 threads, which no launch has."""
    wide = dict(heads=0, q=None, out=None, ldk=D, ldv=D, c=one_head(D), b=batch(rows=rows))
    over = rows * WORKGROUP >= MOST
    if over:
        assert append(L, **wide) == EUNSUPPORTED
        assert read(L, ldk=D, ldv=D, c=one_head(D), b=batch(rows=rows)) == EUNSUPPORTED
    else:   # not refused for its size: what is misaligned is named
        assert append(L, **dict(wide, k=FAKE + 2)) == 3
        assert read(L, ldk=D, ldv=D, c=one_head(D), b=batch(rows=rows), k=FAKE + 2) == 3


def test_bounds_on_rows_times_heads(L):  # noqa: F811
    """As before: 2^26 rows times heads, whatever the workgroups."""
    for heads, kv in ((0, 1), (1, 1), (4, 2), (32, 8)):
        rows = (1 << 26) // (heads + 2 * kv) + 1
        c = cache(kv_heads=kv)
        assert append(L, heads=heads, ldq=heads * 128 or 128, ldo=heads * 128 or 128, ldk=kv * 128, ldv=kv * 128, c=c,
                      b=batch(rows=rows)) == EUNSUPPORTED
        rows = (1 << 26) // (2 * kv) + 1
        assert read(L, ldk=kv * 128, ldv=kv * 128, c=c, b=batch(rows=rows)) == EUNSUPPORTED
    # nothing is launched for no sequence
    assert read(L, b=batch(rows=1 << 25, seqs=0), c=one_head(64), ldk=64, ldv=64) == OK
