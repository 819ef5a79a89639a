"""Limits of the choice of pages that go by the threads of its launches.  Needs no GPU."""
import pytest

from paper_2410_11305_amd import binding as B

A = 4096          # any 16-byte aligned non-null address: rejected before use
MOST = (1 << 24) - 8


@pytest.mark.parametrize("rows,heads", [(MOST + 1, 1), (MOST + 7, 1), ((1 << 23) - 3, 2)])
def test_more_rows_than_a_launch_has_threads_for_are_refused(rows, heads):
    """They are rounded up to a multiple of eight, 256 threads each: 2^32 from here on."""
    assert rows * heads > MOST and rows * heads * 64 * 2 < 2 ** 31 - 1          # (queries and lists fit)
    assert B.kv4_select_workspace_bytes(rows, 1, heads, heads, 1) == 0
    assert B.lib().qspec_kv4_select(A, A, A, A, rows, 1, heads, heads, 64, 64, 4, 9, 1, 0, 1, A, A, 1 << 60, None) == B.ERR_SHAPE


def test_so_many_are_taken():
    assert B.kv4_select_workspace_bytes(MOST, 1, 1, 1, 1) == MOST * 64 * 4
