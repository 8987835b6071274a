"""The recurrent layer's rules that run on the host: what a call may read, without a GPU."""
import ctypes as C

import pytest

from routes import _fn


@pytest.mark.parametrize("tile,J", [(8, 1), (8, 2), (8, 4), (4, 1), (4, 2), (4, 4)])
def test_a_scan_reads_no_position_behind_the_end(tile, J):
    """The walk of a lane's fetches with the kernel's own rules: every position of its own is the one it
    holds when that is computed, and none at or behind the end is read (not even to be discarded)."""
    walk = _fn("_ZN2mt14scan_walk_rowsEiiii", C.c_int, 4)
    for n in range(1, 201):
        for tj in range(J):
            last = walk(n, tile, J, tj)
            assert 0 <= last < n, (n, tj, last)
