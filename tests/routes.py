"""Which form of a kernel a call takes: the library's own rules (host code, no GPU), called by their
C++ names."""
import ctypes as C

from paper_1804_00344_amd import mtstep as mt


def _fn(symbol, restype, nargs):
    f = getattr(mt.lib(), symbol)
    f.restype, f.argtypes = restype, [C.c_int] * nargs
    return f


def attention_form(B, K, S, E, H, A):
    """"beam" or "row": the attention of a step (its scores need rows of 3H + E floats of scratch)."""
    takes = _fn("_ZN2mt20attention_takes_beamEiiiii", C.c_bool, 5)
    return "beam" if S <= 3 * H + E and takes(B, K, S, A, 2 * H) else "row"


def joint_chunks(E, V, M, n=2, bf16=1, num_cu=256):
    """(chunks, chunks per workgroup) of the joint vocabulary pass."""
    f = mt.lib()._ZN2mt18vocab_joint_chunksEiiiiiiPi
    f.restype, f.argtypes = C.c_int, [C.c_int] * 6 + [C.POINTER(C.c_int)]
    group = C.c_int(0)
    return f(bf16, M, V, E, n, num_cu, C.byref(group)), group.value


def encoder_form(B, H, bf16):
    """"fused" (one kernel per position) or "products": a shallow encoder cell without layer norm."""
    return "fused" if _fn("_ZN2mt14enc_step_takesEiii", C.c_bool, 3)(bf16, B, H) else "products"


def vocab_chunks(E, V, M, bf16=1, num_cu=256):
    return _fn("_ZN2mt12vocab_chunksEiiiii", C.c_int, 5)(bf16, M, V, E, num_cu)


class MhaPlan(C.Structure):
    _fields_ = [("tiles", C.c_int), ("parts", C.c_int)] + [(n, C.c_bool) for n in ("step", "few", "share", "sort", "ends")]


def attn_plan(B, S, Hq, Hk, Dh, n_keys, dtype, window=0, num_cu=256):
    """(form, parts of the key axis, whether waves share a tile's keys, masked sentences sorted) of mt_attn_paged or mt_attn_cross;
    the form: "rows" (tiles of four by the vector units), "steps" (tiles of 32 rows) or "tiles" (of 128)."""
    f = mt.lib()._ZN2mt8mha_planEiiiiixibi
    f.restype, f.argtypes = MhaPlan, [C.c_int] * 5 + [C.c_longlong, C.c_int, C.c_bool, C.c_int]
    p = f(Hq, Hk, Dh, B, S, n_keys, window, dtype == "f32", num_cu)
    return "rows" if p.few else "steps" if p.step else "tiles", p.parts, p.share, p.sort


class AppendForm(C.Structure):
    _fields_ = [("tokens", C.c_int), ("stream", C.c_bool)]


def append_form(B, S, Hq, Hk, Dh, dtype, aligned=True, num_cu=256):
    """(positions of a workgroup, whether results are stored past the L2s) of mt_attn_append."""
    f = mt.lib()._ZN2mt11append_formEiiiiiibi
    f.restype, f.argtypes = AppendForm, [C.c_int] * 6 + [C.c_bool, C.c_int]
    r = f(B, S, Hq, Hk, Dh, 4 if dtype == "f32" else 2, aligned, num_cu)
    return r.tokens, r.stream
