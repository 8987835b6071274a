"""The recurrent layer's calls after a call that failed."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_1804_00344_amd import mtstep as mt
from test_gpu_layer import DEV, gen

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def test_a_failed_load_does_not_fail_the_next_call():
    """A matrix of 2^40 bytes fits no card; the call that follows reports its own outcome."""
    W = torch.randn(40, 30, generator=gen(1))
    mat = mt.mt_i8_load(W)
    x, y = torch.randn(5, 40, generator=gen(2)).to(DEV), torch.empty(5, 30, device=DEV)
    ws = torch.empty(mt.mt_i8_workspace_bytes(mat, 5), dtype=torch.uint8, device=DEV)
    h = C.c_void_p()
    assert mt.lib().mt_i8_load(65536, 2 ** 24, W.data_ptr(), None, C.byref(h)) == mt.MT_ERR_OOM and not h.value
    mt.mt_i8_product(mat, x, y, ws)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(y).all())
