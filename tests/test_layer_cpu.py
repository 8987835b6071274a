"""The recurrent layer's entry points without a GPU: what they refuse, on the host, before any launch."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_1804_00344_amd import mtstep as mt
from routes import _fn

P = 1 << 20  # addresses that are never followed: every call below ends before a launch


class I8Head(C.Structure):
    _fields_ = [("magic", C.c_uint32), ("K", C.c_int), ("N", C.c_int), ("Kp", C.c_int), ("Np", C.c_int),
                ("ptrs", C.c_void_p * 3), ("device", C.c_int), ("num_cu", C.c_int)]


class SsmHead(C.Structure):
    _fields_ = [("magic", C.c_uint32), ("cfg", mt.mt_ssm_config), ("Np", C.c_int), ("ptrs", C.c_void_p * 7),
                ("device", C.c_int), ("num_cu", C.c_int)]


def matrix(K, N):
    """A handle of a device that is never the current one: a call with good arguments ends there."""
    return I8Head(0x4d543849, K, N, (K + 127) // 128 * 128, (N + 255) // 256 * 256, (C.c_void_p * 3)(), -2, 256)


def cell(D=64, N=16, G=1, W=4, dtype=mt.MT_BF16):
    return SsmHead(0x4d545353, mt.mt_ssm_config(D, N, G, W, dtype, 1), 16, (C.c_void_p * 7)(), -2, 256)


def status(name, *args):
    return getattr(mt.lib(), name)(*args)


def reached_device_check(rc):
    return rc in (mt.MT_ERR_STATE, mt.MT_ERR_HIP)  # another device is current; or there is none


# ---- loading ------------------------------------------------------------------------------------

@pytest.mark.parametrize("K,N,W,rc", [(0, 4, P, mt.MT_ERR_SHAPE), (65537, 4, P, mt.MT_ERR_SHAPE),
                                      (4, 0, P, mt.MT_ERR_SHAPE), (4, 2 ** 24 + 1, P, mt.MT_ERR_SHAPE),
                                      (4, 4, None, mt.MT_ERR_ARG), (4, 4, P + 2, mt.MT_ERR_ARG)])
def test_i8_load_refuses(K, N, W, rc):
    h = C.c_void_p(7)
    assert status("mt_i8_load", K, N, W, None, C.byref(h)) == rc and not h.value


@pytest.mark.parametrize("kw,rc", [(dict(D=0), mt.MT_ERR_SHAPE), (dict(D=65537), mt.MT_ERR_SHAPE),
                                   (dict(N=0), mt.MT_ERR_SHAPE), (dict(N=257), mt.MT_ERR_SHAPE),
                                   (dict(G=3), mt.MT_ERR_SHAPE), (dict(G=0), mt.MT_ERR_SHAPE),
                                   (dict(W=9), mt.MT_ERR_SHAPE), (dict(W=-1), mt.MT_ERR_SHAPE),
                                   (dict(dtype=2), mt.MT_ERR_DTYPE), (dict(conv_silu=2), mt.MT_ERR_ARG)])
def test_ssm_load_refuses_configurations(kw, rc):
    cfg = mt.mt_ssm_config(8, 4, 1, 2, mt.MT_F32, 0)
    for k, v in kw.items():
        setattr(cfg, k, v)
    h = C.c_void_p(7)
    assert status("mt_ssm_load", C.byref(cfg), C.byref(mt.mt_ssm_weights()), C.byref(h)) == rc and not h.value


@pytest.mark.parametrize("bad", [0.5, float("nan"), float("-inf")])
def test_ssm_load_refuses_rates(bad):
    A = -np.ones((8, 4), np.float32)
    A[3, 2] = bad
    with pytest.raises(mt.MtError) as e:
        mt.mt_ssm_load(mt.make_ssm_config(8, 4), dict(A=A))
    assert e.value.status == mt.MT_ERR_ARG and "A[14]" in str(e.value)


def test_ssm_load_refuses_missing_and_misshapen_parameters():
    A = -np.ones((8, 4), np.float32)
    for w in (dict(), dict(A=A)):  # no A; a convolution without weights
        with pytest.raises(mt.MtError):
            mt.mt_ssm_load(mt.make_ssm_config(8, 4, conv=2), w)
    with pytest.raises(ValueError):
        mt.mt_ssm_load(mt.make_ssm_config(8, 4), dict(A=A, skip=np.ones(7)))


def test_handles_are_checked():
    junk = C.cast((C.c_uint32 * 64)(), C.c_void_p)
    for h in (None, junk):
        assert status("mt_i8_free", h) == mt.MT_ERR_ARG and status("mt_ssm_free", h) == mt.MT_ERR_ARG
        assert status("mt_i8_workspace_bytes", h, 4) == 0 and status("mt_ssm_workspace_bytes", h, 1, 1) == 0
        assert status("mt_i8_product", h, 1, P, 0, 4, P, 0, 4, P, 1 << 40, None) == mt.MT_ERR_ARG
        assert status("mt_ssm_conv", h, 1, 1, None, P, 8, None, P, 8, None, None) == mt.MT_ERR_ARG
        assert status("mt_ssm_conv_step", h, 1, None, 1, P, 8, P, P, 8, P, None) == mt.MT_ERR_ARG
        assert status("mt_ssm_scan", h, 1, 1, None, P, 8, P, 8, P, P, 8, None, 0, None, P, 8, None, P, 1 << 40,
                      None) == mt.MT_ERR_ARG
        assert status("mt_ssm_step", h, 1, None, 1, P, 8, P, 8, P, P, 8, None, 0, P, P, 8, P, None) == mt.MT_ERR_ARG
        assert status("mt_ssm_device_errors", h, C.byref(C.c_int32())) == mt.MT_ERR_ARG


def test_device_errors_of_another_device():
    c = cell()
    assert reached_device_check(status("mt_ssm_device_errors", C.addressof(c), C.byref(C.c_int32())))
    assert status("mt_ssm_device_errors", C.addressof(c), None) == mt.MT_ERR_ARG


# ---- products in 8 bits -------------------------------------------------------------------------

BIG = 1 << 40


def product(**kw):
    w = matrix(kw.pop("K", 100), kw.pop("N", 60))
    a = dict(M=5, x=P, xt=0, ldx=100, y=P * 64, yt=1, ldy=60, ws=P * 512, nb=BIG)
    a.update(kw)
    return status("mt_i8_product", C.addressof(w), a["M"], a["x"], a["xt"], a["ldx"], a["y"], a["yt"], a["ldy"], a["ws"],
                  a["nb"], None)


def test_product_accepts_up_to_the_device_check():
    assert reached_device_check(product())
    assert reached_device_check(product(x=P + 4, ldx=101, y=P * 64 + 2, ldy=77))
    w = matrix(100, 60)
    need = mt.lib().mt_i8_workspace_bytes(C.addressof(w), 5)
    assert need == 256 * 128 + 256 * 4 and reached_device_check(product(nb=need))
    assert product(nb=need - 1) == mt.MT_ERR_WORKSPACE
    # columns of one wider fp32 matrix: 100 columns read, the next 60 written
    assert reached_device_check(product(ldx=160, y=P + 400, yt=0, ldy=160))


@pytest.mark.parametrize("kw,rc", [
    (dict(M=0), mt.MT_ERR_SHAPE), (dict(M=2 ** 24 + 1), mt.MT_ERR_SHAPE), (dict(M=2 ** 24, N=4097, ldy=4097), mt.MT_ERR_SHAPE),
    (dict(xt=2), mt.MT_ERR_DTYPE), (dict(yt=-1), mt.MT_ERR_DTYPE), (dict(x=None), mt.MT_ERR_ARG),
    (dict(y=None), mt.MT_ERR_ARG), (dict(ws=None), mt.MT_ERR_ARG), (dict(x=P + 2), mt.MT_ERR_ARG),
    (dict(y=P * 64 + 1), mt.MT_ERR_ARG), (dict(ws=P * 512 + 16), mt.MT_ERR_ARG), (dict(ldx=99), mt.MT_ERR_SHAPE),
    (dict(ldy=59), mt.MT_ERR_SHAPE), (dict(ldx=-100), mt.MT_ERR_SHAPE), (dict(ldx=2 ** 33), mt.MT_ERR_SHAPE),
    (dict(y=P + 16), mt.MT_ERR_ARG), (dict(ws=P), mt.MT_ERR_ARG), (dict(y=P * 512), mt.MT_ERR_ARG),
    (dict(ldx=160, y=P + 396, yt=0, ldy=160), mt.MT_ERR_ARG)])  # one column shared
def test_product_refuses(kw, rc):
    assert product(**kw) == rc, mt.lib().mt_last_error()


# ---- convolution and scan -----------------------------------------------------------------------

def conv(c=None, **kw):
    c = c or cell()
    a = dict(B=3, S=7, len=None, x=P, ldx=64, si=None, y=P * 64, ldy=64, so=None)
    a.update(kw)
    return status("mt_ssm_conv", C.addressof(c), a["B"], a["S"], a["len"], a["x"], a["ldx"], a["si"], a["y"], a["ldy"],
                  a["so"], None)


def conv_step(c=None, **kw):
    c = c or cell()
    a = dict(M=4, row=None, n=4, x=P, ldx=64, si=P * 128, y=P * 64, ldy=64, so=P * 256)
    a.update(kw)
    return status("mt_ssm_conv_step", C.addressof(c), a["M"], a["row"], a["n"], a["x"], a["ldx"], a["si"], a["y"], a["ldy"],
                  a["so"], None)


def scan(c_=None, **kw):
    c = c_ or cell()
    a = dict(B=3, S=7, len=None, x=P, ldx=64, dt=P * 2, ldd=64, b=P * 4, c=P * 4 + 32, ldbc=32, z=None, ldz=0, si=None,
             y=P * 64, ldy=64, so=None, ws=P * 512, nb=BIG)
    a.update(kw)
    return status("mt_ssm_scan", C.addressof(c), a["B"], a["S"], a["len"], a["x"], a["ldx"], a["dt"], a["ldd"], a["b"], a["c"],
                  a["ldbc"], a["z"], a["ldz"], a["si"], a["y"], a["ldy"], a["so"], a["ws"], a["nb"], None)


def step(c_=None, **kw):
    c = c_ or cell()
    a = dict(M=4, row=None, n=4, x=P, ldx=64, dt=P * 2, ldd=64, b=P * 4, c=P * 4 + 32, ldbc=32, z=None, ldz=0, si=P * 128,
             y=P * 64, ldy=64, so=P * 256)
    a.update(kw)
    return status("mt_ssm_step", C.addressof(c), a["M"], a["row"], a["n"], a["x"], a["ldx"], a["dt"], a["ldd"], a["b"], a["c"],
                  a["ldbc"], a["z"], a["ldz"], a["si"], a["y"], a["ldy"], a["so"], None)


def test_calls_accept_up_to_the_device_check():
    for rc in (conv(), conv(si=P * 8, so=P * 16, len=P * 32), conv(x=P + 2, ldx=65), conv(B=1, S=2 ** 24, y=1 << 45),
               conv_step(), conv_step(so=P * 128), conv_step(row=P * 32, n=2 ** 24, so=1 << 45),
               conv_step(cell(W=1), si=None, so=None), scan(), scan(z=P * 8, ldz=64, si=P * 16, so=P * 32, len=P * 48),
               step(), step(so=P * 128), step(row=P * 32, n=1), step(z=P * 8, ldz=99)):
        assert reached_device_check(rc), mt.lib().mt_last_error()
    # x, dt and y as neighbouring columns of one matrix
    assert reached_device_check(scan(ldx=192, dt=P + 128, ldd=192, y=P + 256, ldy=192))
    c = cell()
    need = mt.lib().mt_ssm_workspace_bytes(C.addressof(c), 3, 7)
    assert need > 0 and reached_device_check(scan(nb=need)) and scan(nb=need - 1) == mt.MT_ERR_WORKSPACE


@pytest.mark.parametrize("kw,rc", [
    (dict(B=0), mt.MT_ERR_SHAPE), (dict(S=0), mt.MT_ERR_SHAPE), (dict(B=4097, S=4096), mt.MT_ERR_SHAPE),
    (dict(ldx=63), mt.MT_ERR_SHAPE), (dict(ldy=0), mt.MT_ERR_SHAPE), (dict(x=None), mt.MT_ERR_ARG),
    (dict(y=None), mt.MT_ERR_ARG), (dict(x=P + 1), mt.MT_ERR_ARG), (dict(len=P + 2), mt.MT_ERR_ARG),
    (dict(si=P * 8 + 8), mt.MT_ERR_ARG), (dict(so=P * 8 + 8), mt.MT_ERR_ARG), (dict(y=P), mt.MT_ERR_ARG),
    (dict(si=P * 8, so=P * 8), mt.MT_ERR_ARG), (dict(so=P), mt.MT_ERR_ARG), (dict(so=P * 64), mt.MT_ERR_ARG)])
def test_prompts_refuse(kw, rc):
    assert conv(**kw) == rc and scan(**kw) == rc, mt.lib().mt_last_error()


@pytest.mark.parametrize("kw,rc", [
    (dict(dt=None), mt.MT_ERR_ARG), (dict(b=None), mt.MT_ERR_ARG), (dict(c=P * 4 + 1), mt.MT_ERR_ARG),
    (dict(ldd=63), mt.MT_ERR_SHAPE), (dict(ldbc=15), mt.MT_ERR_SHAPE), (dict(z=P * 8, ldz=63), mt.MT_ERR_SHAPE),
    (dict(z=P * 64, ldz=64), mt.MT_ERR_ARG), (dict(dt=P * 64), mt.MT_ERR_ARG), (dict(b=P * 64), mt.MT_ERR_ARG)])
def test_scans_refuse(kw, rc):
    assert scan(**kw) == rc and step(**kw) == rc, mt.lib().mt_last_error()


def test_scan_refuses_its_workspace():
    assert scan(ws=None) == mt.MT_ERR_ARG and scan(ws=P * 512 + 16) == mt.MT_ERR_ARG
    assert scan(ws=P) == mt.MT_ERR_ARG and scan(ws=P * 64) == mt.MT_ERR_ARG


@pytest.mark.parametrize("kw,rc", [
    (dict(M=0), mt.MT_ERR_SHAPE), (dict(M=2 ** 24 + 1, n=2 ** 24), mt.MT_ERR_SHAPE), (dict(n=0), mt.MT_ERR_SHAPE),
    (dict(n=3), mt.MT_ERR_SHAPE), (dict(row=P * 32, n=2 ** 24 + 1), mt.MT_ERR_SHAPE), (dict(row=P * 32 + 2), mt.MT_ERR_ARG),
    (dict(si=None), mt.MT_ERR_ARG), (dict(so=None), mt.MT_ERR_ARG), (dict(so=P * 256 + 4), mt.MT_ERR_ARG),
    (dict(row=P * 32, so=P * 128), mt.MT_ERR_ARG),  # gathered states in place
    (dict(so=P * 128 + 64), mt.MT_ERR_ARG), (dict(y=P), mt.MT_ERR_ARG), (dict(ldx=63), mt.MT_ERR_SHAPE)])
def test_tokens_refuse(kw, rc):
    assert conv_step(**kw) == rc and step(**kw) == rc, mt.lib().mt_last_error()


def test_sizes_beyond_the_grids():
    wide = cell(D=65536, W=2)
    assert conv(wide, B=1, S=2 ** 19, ldx=65536, ldy=65536, y=1 << 50) == mt.MT_ERR_SHAPE
    assert conv_step(wide, M=65536, n=65536, ldx=65536, ldy=65536, y=1 << 50) == mt.MT_ERR_SHAPE


def test_no_convolution():
    assert conv(cell(W=0)) == mt.MT_ERR_STATE and conv_step(cell(W=0)) == mt.MT_ERR_STATE


# ---- the binding --------------------------------------------------------------------------------

def test_binding_refuses_tensors():
    rows = lambda t, lead, width, dt=torch.float32: mt._rows(t, "x", lead + (width,), dt, torch.device("cpu"))
    t = torch.zeros(3, 5, 16)
    assert rows(t, (3, 5), 16)[1] == 16 and rows(t[..., 4:12], (3, 5), 8)[1] == 16
    assert rows(torch.zeros(1, 16)[:, :3], (1,), 3)[1] == 3
    for bad in (lambda: rows(t, (3, 5), 15), lambda: rows(t.bfloat16(), (3, 5), 16), lambda: rows(t[:, :4], (3, 4), 16),
                lambda: rows(t[..., ::2], (3, 5), 8), lambda: rows(t.transpose(1, 2), (3, 16), 5),
                lambda: mt._rows(t, "x", (3, 5, 16), t.dtype, torch.device("cuda", 0)),
                lambda: mt._space(t, torch.device("cuda", 0)), lambda: mt._space(t[:, 1:], t.device),
                lambda: mt._packed(t[:, ::2], "s", (3, 3, 16), t.dtype, t.device),
                lambda: mt._packed(torch.zeros(3, dtype=torch.int64), "lens", (3,), torch.int32, t.device)):
        with pytest.raises(ValueError):
            bad()


# ---- which form a call takes ----------------------------------------------------------------------

def i8_form(M, N, K, y_bytes=4, num_cu=256):
    return _fn("_ZN2mt7i8_formEiiiii", C.c_int, 5)(M, N, K, y_bytes, num_cu)


def scan_pieces(B, S, D, N, num_cu=256):
    return _fn("_ZN2mt11scan_piecesEiiiii", C.c_int, 5)(B, S, D, N, num_cu)


@pytest.mark.parametrize("M,N,K,form", [(1, 50000, 512, -1), (4, 2048, 4096, -1), (5, 2048, 512, 0), (4, 2048, 4097, 0),
                                        (64, 2048, 2048, 0), (4096, 512, 2048, 1), (128, 50000, 512, 2), (768, 50000, 512, 3),
                                        (512, 8192, 2048, 2), (8192, 8192, 4096, 4)])
def test_product_form(M, N, K, form):
    assert i8_form(M, N, K, 2 if K == 4096 else 4) == form


def test_gpu_product_cases_take_every_form():
    from test_gpu_layer import LARGE_PRODUCTS, PRODUCTS
    cases = [(M, N, K) for M, K, N, *_ in PRODUCTS] + [(M, N, K) for M, K, N in LARGE_PRODUCTS]
    assert {i8_form(M, N, K, es) for M, N, K in cases for es in (2, 4)} == {-1, 0, 1, 2, 3, 4}


@pytest.mark.parametrize("B,S,D,N,pieces", [(64, 80, 2048, 16, 1), (1, 8, 2048, 16, 1), (1, 8192, 2048, 16, 64),
                                            (1, 2 ** 20, 64, 16, 256), (1, 4, 65536, 256, 1)])
def test_scan_pieces(B, S, D, N, pieces):
    assert scan_pieces(B, S, D, N) == pieces


def test_scan_pieces_cover_the_axis_and_the_workspace_holds_them():
    for S in (1, 15, 16, 17, 100, 1000, 12345):
        n = scan_pieces(2, S, 100, 24)
        assert 1 <= n <= (S + 7) // 8  # pieces of whole tiles of 8 positions, the last one shorter
        c = cell(D=100, N=24)
        assert mt.lib().mt_ssm_workspace_bytes(C.addressof(c), 2, S) == 2 * (n - 1) * 100 * 33 * 4 + 256


def test_gpu_scan_cases_take_both_forms():
    from test_gpu_layer import SCANS
    pieces = [scan_pieces(B, S, D, N) for B, S, D, N, *_ in SCANS]
    assert min(pieces) == 1 and max(pieces) >= 16
