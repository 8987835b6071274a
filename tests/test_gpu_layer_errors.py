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


def test_a_matrix_of_another_device_is_waited_for(monkeypatch):
    """With another device current the load would read the matrix while its own device may still write it."""
    waited = []
    monkeypatch.setattr(torch.cuda, "synchronize", waited.append)
    W = torch.randn(8, 4, device=DEV)
    mt._host_or_device(W)
    assert waited == []
    monkeypatch.setattr(mt, "_current_device", lambda: torch.device("cuda", 1))
    _, p = mt._host_or_device(W)
    assert waited == [W.device] and p == W.data_ptr()
    mt._host_or_device(W.cpu())
    assert len(waited) == 1
