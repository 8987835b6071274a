"""The attention layer's entry points without a GPU: what they refuse, on the host, before any launch; which form a call
takes; and the definitions that the GPU tests compare with, against plainer ones."""
import ctypes as C
import math

import pytest
import torch

import attn_ref as ref
from paper_1804_00344_amd import mtstep as mt
from routes import _fn
from test_layer_cpu import BIG, P, reached_device_check, status


class AttnHead(C.Structure):
    _fields_ = [("magic", C.c_uint32), ("cfg", mt.mt_attn_config), ("page_log2", C.c_int), ("scale2", C.c_float),
                ("ptrs", C.c_void_p * 5), ("device", C.c_int), ("num_cu", C.c_int)]


def layer(Hq=8, Hk=4, Dh=64, page=16, dtype="bf16", **kw):
    """A handle of a device that is never the current one: a call with good arguments ends there."""
    return AttnHead(0x4d544154, mt.make_attn_config(Hq, Hk, Dh, page=page, dtype=dtype, **kw), page.bit_length() - 1, 0.1,
                    (C.c_void_p * 5)(), -2, 256)


# ---- loading ------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw,rc", [
    (dict(Hq=0), mt.MT_ERR_SHAPE), (dict(Hq=1025, Hk=1), mt.MT_ERR_SHAPE), (dict(Hk=3), mt.MT_ERR_SHAPE), (dict(Hk=0), mt.MT_ERR_SHAPE),
    (dict(Hk=16), mt.MT_ERR_SHAPE), (dict(Dh=0), mt.MT_ERR_SHAPE), (dict(Dh=60), mt.MT_ERR_SHAPE), (dict(Dh=264), mt.MT_ERR_SHAPE),
    (dict(Hq=1024, Hk=1, Dh=72), mt.MT_ERR_SHAPE), (dict(page=4), mt.MT_ERR_SHAPE), (dict(page=24), mt.MT_ERR_SHAPE),
    (dict(page=512), mt.MT_ERR_SHAPE), (dict(window=-1), mt.MT_ERR_SHAPE), (dict(rot=7), mt.MT_ERR_SHAPE), (dict(rot=66), mt.MT_ERR_SHAPE),
    (dict(scale=-1.0), mt.MT_ERR_ARG), (dict(scale=float("inf")), mt.MT_ERR_ARG), (dict(scale=float("nan")), mt.MT_ERR_ARG),
    (dict(qk_norm=True, norm_eps=-1.0), mt.MT_ERR_ARG), (dict(rot=8, rot_base=0.0), mt.MT_ERR_ARG),
    (dict(rot=8, rot_base=float("nan")), mt.MT_ERR_ARG)])
def test_load_refuses_configurations(kw, rc):
    cfg = mt.make_attn_config(**{**dict(Hq=8, Hk=4, Dh=64), **kw})
    with pytest.raises(mt.MtError) as e:
        mt.mt_attn_load(cfg)
    assert e.value.status == rc


def test_load_refuses_a_scale_that_is_infinite_in_powers_of_two():
    """Scores are held times log2(e): a product of such a scale with a zero would be no number."""
    for scale, ok in ((3e38, False), (2.4e38, False), (2.3e38, True)):
        try:
            mt.mt_attn_load(mt.make_attn_config(8, 4, 64, scale=scale))
        except mt.MtError as e:  # a good one ends where there is no device
            assert (e.status != mt.MT_ERR_ARG) == ok
        else:
            assert ok


def test_load_refuses_flags_types_and_parameters():
    for field, v, rc in (("dtype", 2, mt.MT_ERR_DTYPE), ("qk_norm", 2, mt.MT_ERR_ARG), ("rot_pairs", -1, mt.MT_ERR_ARG)):
        cfg = mt.make_attn_config(8, 4, 64)
        setattr(cfg, field, v)
        with pytest.raises(mt.MtError) as e:
            mt.mt_attn_load(cfg)
        assert e.value.status == rc
    cfg = mt.make_attn_config(8, 4, 64, rot=8, qk_norm=True)
    for w in (dict(gq=torch.ones(63)), dict(freq=torch.ones(5))):
        with pytest.raises(ValueError):
            mt.mt_attn_load(cfg, w)
    with pytest.raises(mt.MtError) as e:
        mt.mt_attn_load(cfg, dict(freq=torch.tensor([1.0, 1.0, float("inf"), 1.0])))
    assert e.value.status == mt.MT_ERR_ARG and "freq[2]" in str(e.value)
    assert status("mt_attn_load", None, None, C.byref(C.c_void_p())) == mt.MT_ERR_ARG
    assert status("mt_attn_load", C.byref(cfg), None, None) == mt.MT_ERR_ARG


def test_handles_are_checked():
    junk = C.cast((C.c_uint32 * 64)(), C.c_void_p)
    for h in (None, junk):
        assert status("mt_attn_free", h) == mt.MT_ERR_ARG and status("mt_attn_workspace_bytes", h, 1, 1, 1) == 0
        assert status("mt_pages_workspace_bytes", h, 1, 1) == 0
        assert append(h) == paged(h) == cross(h) == advance(h) == pack(h) == mt.MT_ERR_ARG
        assert status("mt_attn_device_errors", h, C.byref(C.c_int32())) == mt.MT_ERR_ARG
    a = layer()
    assert reached_device_check(status("mt_attn_device_errors", C.addressof(a), C.byref(C.c_int32())))
    assert status("mt_attn_device_errors", C.addressof(a), None) == mt.MT_ERR_ARG


# ---- calls: addresses that are never followed ----------------------------------------------------------

def _call(name, order, base, a, kw):
    base = {**base, **kw}
    handle = layer() if a == "new" else a
    at = C.addressof(handle) if isinstance(handle, AttnHead) else handle
    return status(name, at, *[base[k] for k in order.split()], None)


def append(a="new", **kw):
    return _call("mt_attn_append", "B S n len q ldq k ldk v ldv o ldo t nb np kp vp",
                 dict(B=3, S=7, n=None, len=P, q=P * 2, ldq=512, k=P * 3, ldk=256, v=P * 4, ldv=256, o=P * 5, ldo=512, t=P * 6, nb=4,
                      np=10, kp=P * 8, vp=P * 16), a, kw)


def paged(a="new", **kw):
    return _call("mt_attn_paged", "B S n len q ldq t nb np kp vp y ldy ws wb",
                 dict(B=3, S=7, n=None, len=P, q=P * 2, ldq=512, t=P * 6, nb=4, np=10, kp=P * 8, vp=P * 16, y=P * 5, ldy=512,
                      ws=P * 512, wb=BIG), a, kw)


def cross(a="new", **kw):
    return _call("mt_attn_cross", "B T n S mask q ldq k ldk v ldv y ldy ws wb",
                 dict(B=3, T=7, n=None, S=9, mask=None, q=P * 2, ldq=512, k=P * 3, ldk=256, v=P * 4, ldv=256, y=P * 5, ldy=512,
                      ws=P * 512, wb=BIG), a, kw)


def advance(a="new", **kw):
    return _call("mt_pages_advance", "Mi M row add ti li nb np to lo fo layers k v ws wb",
                 dict(Mi=4, M=4, row=None, add=None, ti=P, li=P * 2, nb=4, np=10, to=P * 3, lo=P * 4, fo=None, layers=2, k=P * 8,
                      v=P * 16, ws=P * 512, wb=BIG), a, kw)


def pack(a="new", **kw):
    return _call("mt_pages_pack", "M ti li nb np layers ki vi no to lo uo ko vo ws wb",
                 dict(M=4, ti=P, li=P * 2, nb=4, np=10, layers=2, ki=P * 8, vi=P * 16, no=5, to=P * 3, lo=P * 4, uo=None, ko=P * 32,
                      vo=P * 64, ws=P * 512, wb=BIG), a, kw)


def test_calls_accept_up_to_the_device_check():
    for rc in (append(), append(o=P * 2), append(n=P * 7, q=P * 2 + 2, ldq=513), append(q=P * 2, ldq=1024, k=P * 2 + 1024, ldk=1024),
               paged(), paged(n=P * 7, y=P * 5 + 2, ldy=600), paged(layer(window=5)), cross(), cross(mask=P * 7, n=P * 9),
               cross(k=P * 3, ldk=512, v=P * 3 + 512, ldv=512), advance(), advance(row=P * 5, add=P * 6, fo=P * 7, M=9),
               pack(), pack(uo=P * 7, no=2 ** 24, ko=1 << 50, vo=1 << 51)):
        assert reached_device_check(rc), mt.lib().mt_last_error()
    a = layer()
    for call, need in ((paged, mt.lib().mt_attn_workspace_bytes(C.addressof(a), 3, 7, 64)),
                       (cross, mt.lib().mt_attn_workspace_bytes(C.addressof(a), 3, 7, 9)),
                       (advance, mt.lib().mt_pages_workspace_bytes(C.addressof(a), 4, 10))):
        assert need > 0 and reached_device_check(call(wb=need)) and call(wb=need - 1) == mt.MT_ERR_WORKSPACE


A, SH = mt.MT_ERR_ARG, mt.MT_ERR_SHAPE


@pytest.mark.parametrize("kw,rc", [
    (dict(B=0), SH), (dict(S=0), SH), (dict(B=4097, S=4096), SH), (dict(nb=0), SH), (dict(nb=2 ** 27), SH), (dict(np=0), SH),
    (dict(np=2 ** 24 + 1), SH), (dict(B=2 ** 20, S=1, nb=2 ** 11), SH), (dict(len=None), A), (dict(len=P + 2), A), (dict(n=P + 1), A),
    (dict(t=None), A), (dict(t=P + 2), A), (dict(q=None), A), (dict(q=P + 1), A), (dict(ldq=511), SH), (dict(kp=None), A),
    (dict(kp=P * 8 + 8), A), (dict(vp=P * 16 + 4), A), (dict(vp=None), A)])
def test_new_positions_refuse(kw, rc):
    assert append(**kw) == rc and paged(**kw) == rc, mt.lib().mt_last_error()


@pytest.mark.parametrize("kw,rc", [
    (dict(k=None), A), (dict(v=P + 1), A), (dict(ldk=255), SH), (dict(ldv=0), SH), (dict(ldo=511), SH), (dict(o=None), A),
    (dict(o=P * 3), A), (dict(o=P * 2, ldo=600), A), (dict(o=P * 2 + 1024, ldo=512), A), (dict(kp=P * 2), A), (dict(vp=P * 8), A),
    (dict(kp=P * 6), A), (dict(vp=P), A), (dict(o=P * 2, kp=P * 2), A)])
def test_append_refuses(kw, rc):
    assert append(**kw) == rc, mt.lib().mt_last_error()


@pytest.mark.parametrize("kw,rc", [(dict(y=None), A), (dict(y=P + 1), A), (dict(ldy=511), SH), (dict(ws=None), A),
                                   (dict(ws=P * 512 + 16), A), (dict(y=P * 2), A), (dict(ws=P * 2), A), (dict(y=P * 512), A)])
def test_attention_refuses(kw, rc):
    assert paged(**kw) == rc and cross(**kw) == rc, mt.lib().mt_last_error()
    assert paged(y=P * 8) == paged(y=P * 6) == paged(ws=P * 16) == A


@pytest.mark.parametrize("kw,rc", [(dict(B=0), SH), (dict(T=0), SH), (dict(S=0), SH), (dict(B=2 ** 14, S=2 ** 11), SH), (dict(k=None), A),
                                   (dict(v=P * 4 + 1), A), (dict(ldk=255), SH), (dict(mask=P + 2), A), (dict(y=P * 3), A),
                                   (dict(n=P + 2), A), (dict(mask=P * 5), A)])
def test_cross_refuses(kw, rc):
    assert cross(**kw) == rc, mt.lib().mt_last_error()


@pytest.mark.parametrize("kw,rc", [
    (dict(M=0), SH), (dict(M=2 ** 20 + 1), SH), (dict(nb=0), SH), (dict(np=0), SH), (dict(layers=0), SH), (dict(layers=1025), SH),
    (dict(ti=None), A), (dict(li=P + 1), A), (dict(to=None), A), (dict(lo=None), A), (dict(ws=None), A), (dict(to=P), A), (dict(lo=P * 2), A),
    (dict(ws=P), A), (dict(lo=P * 3 + 4), A)])
def test_tables_refuse(kw, rc):
    assert advance(**kw, **(dict(Mi=kw["M"]) if "M" in kw else {})) == rc and pack(**kw) == rc, mt.lib().mt_last_error()


@pytest.mark.parametrize("kw,rc", [
    (dict(Mi=5), SH), (dict(Mi=0, row=P * 5), SH), (dict(row=P + 2), A), (dict(add=P + 2), A), (dict(fo=P + 2), A), (dict(k=None), A),
    (dict(v=P * 16 + 8), A), (dict(v=P * 8), A), (dict(row=P * 3), A), (dict(add=P * 4), A), (dict(fo=P * 4 + 4), A), (dict(k=P), A)])
def test_advance_refuses(kw, rc):
    assert advance(**kw) == rc, mt.lib().mt_last_error()


@pytest.mark.parametrize("kw,rc", [(dict(no=0), SH), (dict(no=2 ** 24 + 1), SH), (dict(ki=None), A), (dict(vo=None), A), (dict(ko=P * 8), A),
                                   (dict(vo=P * 16), A), (dict(ko=P * 64), A), (dict(uo=P * 4), A), (dict(uo=P + 1), A)])
def test_pack_refuses(kw, rc):
    assert pack(**kw) == rc, mt.lib().mt_last_error()


def test_sizes_beyond_the_heads():
    wide = layer(Hq=1024, Hk=1, Dh=64)
    assert paged(wide, B=2 ** 21, S=1, ldq=65536, ldy=65536, y=1 << 50) == SH
    assert mt.lib().mt_attn_workspace_bytes(C.addressof(wide), 2 ** 21, 1, 10) == 0
    assert mt.lib().mt_attn_workspace_bytes(C.addressof(wide), 1, 1, 2 ** 30 + 1) == 0


def test_append_takes_any_number_of_heads_in_all():
    wide = layer(Hq=1024, Hk=1, Dh=64)
    big = dict(B=2 ** 21, S=1, q=1 << 49, ldq=65536, o=1 << 50, ldo=65536, k=1 << 51, v=1 << 52, t=1 << 53, len=1 << 54)
    assert reached_device_check(append(wide, **big)), mt.lib().mt_last_error()
    assert append(wide, **{**big, "B": 2 ** 24 + 1}) == SH


# ---- the definitions --------------------------------------------------------------------------------

def test_reference_attention_is_the_sum_over_seen_keys():
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(n, 6, generator=g).double() for n in (5, 9, 9))
    seen = ref.causal(2, 5, 9, 3)
    k[8], v[8] = float("nan"), float("inf")  # seen by none
    y, _ = ref.attention(q, k, v, seen, 0.7)
    for i in range(5):
        js = [j for j in range(9) if i + 2 - 3 < j <= i + 2]
        w = [math.exp(0.7 * float(q[i] @ k[j])) for j in js]
        want = sum(a * v[j] for a, j in zip(w, js)) / sum(w)
        assert float((y[i] - want).abs().max()) < 1e-12
    none, _ = ref.attention(q, k, v, torch.zeros(5, 9, dtype=torch.bool), 0.7)
    assert bool((none == 0).all())


def test_reference_rotation_keeps_lengths_and_differences():
    x = torch.randn(2, 8, generator=torch.Generator().manual_seed(2)).double()
    f = torch.tensor([1.0, 0.3, 0.01, 0.0001], dtype=torch.float64)
    for pairs in (False, True):
        at = lambda p: ref.turn_heads(x, torch.tensor([p, p + 5]), 8, False, 0, None, 8, pairs, f)[0]
        assert abs(float(at(3)[0].norm() - x[0].norm())) < 1e-12
        assert abs(float(at(3)[0] @ at(3)[1]) - float(at(40)[0] @ at(40)[1])) < 1e-12  # the product of two turns


def test_reference_tables():
    rows = [(10, [3, 1]), (16, [0, 2])]
    tables, lens, free, copies = ref.advance(rows, [0, 0, 1, -1], [1, 1, 1, 9], 8, 4, 10)
    assert tables == [[3, 4], [3, 1], [0, 2, 5], [6, 7]] and lens == [11, 11, 17, 9] and free == 2 and copies == [(1, 4, 2)]
    assert ref.advance(rows, [0, 1], [1, 1], 8, 2, 10) is None  # 17 positions of 16
    assert ref.advance(rows, [0, 0], [1, 1], 8, 4, 5) is not None and ref.advance(rows, [0, 0, 1], [1, 1, 0], 8, 4, 4) is None
    assert ref.pack([(9, [7, 2]), (8, [7, 0])], 8) == ([[1, 0], [1]], [2, 7])
