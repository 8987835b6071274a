"""The recurrent layer's rules that run on the host: what a call may read, without a GPU."""
import ctypes as C

import pytest

from paper_1804_00344_amd import mtstep as mt
from routes import _fn
from test_layer_cpu import cell, conv, conv_step, matrix, product, reached_device_check, scan, step


@pytest.mark.parametrize("tile,J", [(8, 1), (8, 2), (8, 4), (4, 1), (4, 2), (4, 4)])
def test_a_scan_reads_no_position_behind_the_end(tile, J):
    """The walk of a lane's fetches with the kernel's own rules: every position of its own is the one it
    holds when that is computed, and none at or behind the end is read (not even to be discarded)."""
    walk = _fn("_ZN2mt14scan_walk_rowsEiiii", C.c_int, 4)
    for n in range(1, 201):
        for tj in range(J):
            last = walk(n, tile, J, tj)
            assert 0 <= last < n, (n, tj, last)


def test_a_workspace_for_a_size_that_is_refused():
    """The sizes of the header: the call refuses what is larger, and its workspace is 0 bytes as for any bad input."""
    wide, need = cell(D=65536, W=2), mt.lib().mt_ssm_workspace_bytes
    far = dict(B=1, ldx=65536, ldd=65536, ldy=65536, dt=1 << 44, b=1 << 46, c=(1 << 46) + 32, y=1 << 50, ws=1 << 52, nb=1 << 60)
    assert need(C.addressof(wide), 1, 2 ** 18) > 0 and reached_device_check(scan(wide, S=2 ** 18, **far))
    assert need(C.addressof(wide), 1, 2 ** 18 + 1) == 0 and scan(wide, S=2 ** 18 + 1, **far) == mt.MT_ERR_SHAPE
    m, need = matrix(100, 2 ** 20), mt.lib().mt_i8_workspace_bytes
    far = dict(N=2 ** 20, ldy=2 ** 20, y=1 << 50, ws=1 << 56, nb=1 << 60)
    assert need(C.addressof(m), 2 ** 16) > 0 and reached_device_check(product(M=2 ** 16, **far))
    assert need(C.addressof(m), 2 ** 16 + 1) == 0 and product(M=2 ** 16 + 1, **far) == mt.MT_ERR_SHAPE


@pytest.mark.parametrize("ld,rc", [(2 ** 32, None), (2 ** 32 + 1, mt.MT_ERR_SHAPE)])
def test_the_largest_row_stride(ld, rc):
    got = conv(ldx=ld, y=1 << 50), scan(ldx=ld, dt=1 << 44, b=1 << 46, c=(1 << 46) + 32, y=1 << 50, ws=1 << 52), \
        step(ldx=ld, dt=1 << 44, b=1 << 46, c=(1 << 46) + 32, si=1 << 47, y=1 << 50, so=1 << 48), \
        conv_step(ldx=ld, si=1 << 47, y=1 << 50, so=1 << 48), product(ldx=ld, y=1 << 50, ws=1 << 56)
    for r in got:
        assert reached_device_check(r) if rc is None else r == rc, mt.lib().mt_last_error()
