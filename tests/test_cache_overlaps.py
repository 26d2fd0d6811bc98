"""Arrays of the paged cache's calls that overlap, refused before anything is launched (no GPU; the pointers are made
up and never read)."""
import pytest

from test_cache_refusals import INVALID, UNSUPPORTED, P, addr, kv, mcd     # noqa: F401  (mcd: the fixture)

N, COLS, KEEP = 3, 4, 5                                     # sequences, table columns, most kept


def compact_call(mcd, len_out, table=P, out=2 * P, start=3 * P, keep=4 * P, n_keep=5 * P):
    """Of more layers than a call takes: nothing is launched, whatever the arrays."""
    k = kv(mcd, n_layers=40000)
    return mcd.load_library().mcd_pages_compact(addr(k), N, table, out, COLS, start, keep, KEEP, n_keep, len_out, P, None)


@pytest.mark.parametrize("name,n", [("table", N * COLS), ("out", N * COLS), ("start", N), ("keep", N * KEEP), ("n_keep", N)])
def test_compact_lengths_overlap_an_input(mcd, name, n):     # noqa: F811
    """The length that one CTA writes is what others have yet to read: len_out is an array of its own."""
    at = 100 * P
    for len_out in (at, at + 4 * (n - 1), at - 4 * (N - 1)):  # the same, its last and its first element
        assert compact_call(mcd, len_out, **{name: at}) == INVALID
    for len_out in (None, at + 4 * n, at - 4 * N):            # none, right behind it, right before it
        assert compact_call(mcd, len_out, **{name: at}) == UNSUPPORTED


def test_compact_in_place_lengths_overlap_the_table(mcd):    # noqa: F811
    assert compact_call(mcd, 100 * P, table=100 * P, out=100 * P) == INVALID
    assert compact_call(mcd, 99 * P, table=100 * P, out=100 * P) == UNSUPPORTED
