"""ctypes binding of libmtstep (declarations in include/mtstep.h).

Argument marshalling only: every step of the decoder runs in the library's HIP
kernels.  Device buffers are passed as torch tensors (or raw integer device
addresses); streams as torch streams (default: torch's current stream).  The
binding raises if the built library is missing — there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional

import numpy as np

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libmtstep.so")

MT_OK, MT_ERR_ARG, MT_ERR_SHAPE, MT_ERR_DTYPE, MT_ERR_HIP, MT_ERR_OOM, MT_ERR_STATE, MT_ERR_WORKSPACE = (
    0, -1, -2, -3, -4, -5, -6, -7)
MT_F32, MT_BF16 = 0, 1
KERNELS = ["GEMM_GRU1", "GRU_CELL", "GEMM_S1", "ATTENTION", "GEMM_CTX", "GEMM_READOUT", "READOUT",
           "VOCAB_GEMM", "LSE", "TOPK", "PRECOMPUTE", "VOCAB_THRESHOLD", "GEMM_TRANSITION", "ENSEMBLE",
           "BEAM_FINISH", "ENCODE"]
KERNEL_ID = {n: i for i, n in enumerate(KERNELS)}


class MtError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"libmtstep status {status}: {msg}")
        self.status = status


class mt_config(C.Structure):
    _fields_ = [("E", C.c_int32), ("H", C.c_int32), ("A", C.c_int32), ("V", C.c_int32),
                ("layer_norm", C.c_int32), ("tied_output", C.c_int32), ("k_max", C.c_int32),
                ("gemm_dtype", C.c_int32), ("ln_eps", C.c_float), ("dec_transitions", C.c_int32),
                ("src_V", C.c_int32), ("dual_source", C.c_int32), ("enc_transitions", C.c_int32),
                ("enc_layer_norm", C.c_int32)]


WEIGHT_FIELDS = ["emb", "W1", "U1", "b1", "Ua", "ba", "Wa", "va", "W2", "U2", "b2", "Wt_s", "Wt_y",
                 "Wt_c", "bt", "Wo", "bo", "Wi", "bi", "g1a", "be1a", "g1u", "be1u", "g2a", "be2a",
                 "g2u", "be2u", "gt", "bet", "Ut", "btr", "gtu", "betu",
                 "semb", "Wef", "Uef", "bef", "Web", "Ueb", "beb", "Ua2", "ba2", "Wa2", "va2",
                 "Utef", "btef", "Uteb", "bteb", "gea", "bea", "geu", "beu", "gteu", "beteu"]

_fp = C.POINTER(C.c_float)


class mt_weights(C.Structure):
    _fields_ = [(n, _fp) for n in WEIGHT_FIELDS]


class mt_taps(C.Structure):
    _fields_ = [("s1", C.c_void_p), ("c", C.c_void_p), ("t", C.c_void_p)]


class mt_ssm_config(C.Structure):
    _fields_ = [("D", C.c_int32), ("N", C.c_int32), ("G", C.c_int32), ("W", C.c_int32), ("dtype", C.c_int32),
                ("conv_silu", C.c_int32)]


SSM_WEIGHT_FIELDS = ["A", "dt_bias", "skip", "conv_w", "conv_b"]


class mt_ssm_weights(C.Structure):
    _fields_ = [(n, _fp) for n in SSM_WEIGHT_FIELDS]


_lib = None
_vp = C.c_void_p


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        # The library must run on torch's HIP runtime: its device pointers and streams are
        # torch's.  torch's runtime carries the soname libamdhip64.so.7 but torch names it
        # libamdhip64.so, so loading libmtstep first would bring in a second runtime (the one
        # libmtstep was linked against), which then fails to initialise beside torch's.  With
        # torch loaded first, libmtstep's dependency resolves to the runtime already there.
        import torch  # noqa: F401
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                               "(python -m paper_1804_00344_amd.build)")
        L = C.CDLL(LIB_PATH)
        L.mt_last_error.restype = C.c_char_p
        L.mt_last_error.argtypes = []
        L.mt_load_weights.argtypes = [C.POINTER(mt_config), C.POINTER(mt_weights), C.POINTER(_vp)]
        L.mt_free.argtypes = [_vp]
        L.mt_workspace_bytes.argtypes = [_vp, C.c_int, C.c_int, C.c_int]
        L.mt_workspace_bytes.restype = C.c_size_t
        L.mt_precompute_ctx.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, _vp, _vp, _vp, C.c_size_t, _vp]
        L.mt_precompute_ctx_noalloc.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, _vp, _vp, _vp]
        L.mt_precompute_ctx_noalloc.restype = C.c_int
        L.mt_decoder_step.argtypes = [_vp, C.c_int, C.c_int, C.c_int, _vp, _vp, C.c_int, _vp, _vp, _vp,
                                      _vp, _vp, _vp, _vp, C.POINTER(mt_taps), _vp, C.c_size_t, _vp]
        L.mt_beam_topk.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, _vp, _vp, _vp, _vp, _vp, C.c_size_t, _vp]
        L.mt_device_errors.argtypes = [_vp, C.POINTER(C.c_int32)]
        L.mt_ensemble_logp.argtypes = [_vp, C.c_int, C.POINTER(_vp), C.POINTER(C.c_float), C.c_int, _vp, _vp]
        L.mt_precompute_keys2.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, _vp, _vp, C.c_size_t, _vp]
        L.mt_decoder_step_dual.argtypes = [_vp, C.c_int, C.c_int, C.c_int, _vp, _vp, C.c_int, _vp, _vp, _vp, _vp,
                                           C.c_int, _vp, _vp, _vp, _vp, _vp, _vp, C.POINTER(mt_taps), _vp,
                                           C.c_size_t, _vp]
        L.mt_encode_workspace_bytes.argtypes = [_vp, C.c_int, C.c_int]
        L.mt_encode_workspace_bytes.restype = C.c_size_t
        L.mt_encode.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, _vp, _vp, C.c_size_t, _vp]
        L.mt_beam_finish.argtypes = [_vp, C.c_int, C.c_int, C.c_int, C.c_int32, C.c_float, C.c_int] + [_vp] * 14
        L.mt_profile_enable.argtypes = [_vp, C.c_uint32]
        L.mt_profile_reset.argtypes = [_vp]
        L.mt_profile_sample.argtypes = [_vp, C.c_uint32]
        L.mt_profile_sample.restype = C.c_int
        L.mt_profile_query.argtypes = [_vp, C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        L.mt_ensemble_step.argtypes = [_vp, C.c_int, C.c_int, C.c_float, C.c_int, C.c_int, C.c_int, _vp, _vp, C.c_int, _vp,
                                       _vp, _vp, _vp, _vp, _vp, _vp, C.c_size_t, _vp]
        L.mt_ensemble_step.restype = C.c_int
        L.mt_ensemble_topk.argtypes = [C.c_int, C.POINTER(_vp), C.POINTER(C.c_float), C.POINTER(_vp),
                                       C.POINTER(C.c_size_t), C.c_int, C.c_int, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
        L.mt_ensemble_topk.restype = C.c_int
        L.mt_beam_nbest.argtypes = [_vp, C.c_int, C.c_int, C.c_int] + [_vp] * 9 + [C.c_int, _vp]
        L.mt_beam_nbest.restype = C.c_int
        L.mt_set_state_reuse.argtypes = [_vp, C.c_int]
        L.mt_set_state_reuse.restype = C.c_int
        L.mt_ensemble_joint_ok.argtypes = [C.c_int, C.POINTER(_vp)]
        L.mt_ensemble_joint_ok.restype = C.c_int
        L.mt_recomputed_rows.argtypes = [_vp, C.POINTER(C.c_int64)]
        L.mt_recomputed_rows.restype = C.c_int
        i64, sz = C.c_int64, C.c_size_t
        L.mt_i8_load.argtypes = [C.c_int, C.c_int, _vp, _vp, C.POINTER(_vp)]
        L.mt_i8_free.argtypes = [_vp]
        L.mt_i8_workspace_bytes.argtypes = [_vp, C.c_int]
        L.mt_i8_workspace_bytes.restype = sz
        L.mt_i8_product.argtypes = [_vp, C.c_int, _vp, C.c_int, i64, _vp, C.c_int, i64, _vp, sz, _vp]
        L.mt_ssm_load.argtypes = [C.POINTER(mt_ssm_config), C.POINTER(mt_ssm_weights), C.POINTER(_vp)]
        L.mt_ssm_free.argtypes = [_vp]
        L.mt_ssm_workspace_bytes.argtypes = [_vp, C.c_int, C.c_int]
        L.mt_ssm_workspace_bytes.restype = sz
        L.mt_ssm_conv.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, i64, _vp, _vp, i64, _vp, _vp]
        L.mt_ssm_conv_step.argtypes = [_vp, C.c_int, _vp, C.c_int, _vp, i64, _vp, _vp, i64, _vp, _vp]
        L.mt_ssm_scan.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, i64, _vp, i64, _vp, _vp, i64, _vp, i64, _vp, _vp,
                                  i64, _vp, _vp, sz, _vp]
        L.mt_ssm_step.argtypes = [_vp, C.c_int, _vp, C.c_int, _vp, i64, _vp, i64, _vp, _vp, i64, _vp, i64, _vp, _vp,
                                  i64, _vp, _vp]
        L.mt_ssm_device_errors.argtypes = [_vp, C.POINTER(C.c_int32)]
        for f in ("mt_i8_load", "mt_i8_free", "mt_i8_product", "mt_ssm_load", "mt_ssm_free", "mt_ssm_conv",
                  "mt_ssm_conv_step", "mt_ssm_scan", "mt_ssm_step", "mt_ssm_device_errors"):
            getattr(L, f).restype = C.c_int
        L.mt_round_bf16.argtypes = [_vp, _vp, C.c_size_t]
        L.mt_round_bf16.restype = None
        for f in ("mt_load_weights", "mt_free", "mt_precompute_ctx", "mt_decoder_step", "mt_beam_topk",
                  "mt_ensemble_logp", "mt_beam_finish", "mt_encode", "mt_precompute_keys2", "mt_decoder_step_dual",
                  "mt_device_errors", "mt_profile_enable", "mt_profile_reset", "mt_profile_query"):
            getattr(L, f).restype = C.c_int
        _lib = L
    return _lib


def mt_round_bf16(x: np.ndarray) -> np.ndarray:
    """bf16 bit patterns (uint16) of fp32 values, as mt_load_weights converts a bf16 model's
    matrices (host memory, no device)."""
    src = np.ascontiguousarray(x, np.float32)
    dst = np.empty(src.shape, np.uint16)
    lib().mt_round_bf16(src.ctypes.data, dst.ctypes.data, src.size)
    return dst


def _check(rc: int):
    if rc != MT_OK:
        raise MtError(rc, lib().mt_last_error().decode())


def _ptr(x) -> Optional[int]:
    """Device address of a torch tensor (contiguous), an int, or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if not x.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return x.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


_raw_stream = None


def _stream_on(stream, device) -> Optional[int]:
    """The same, of a given device: the call that torch's own generated code makes for it takes 0.1 us, building
    a stream object 2.5, where a launch takes 4."""
    global _raw_stream
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    if _raw_stream is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda i: torch.cuda.current_stream(i).cuda_stream)
        torch.cuda.init()
    return _raw_stream(device.index)


def make_config(E, H, A, V, *, layer_norm=False, tied_output=False, k_max=16, gemm="f32", ln_eps=1e-5,
                transitions=0, src_V=0, dual_source=False, enc_transitions=0, enc_layer_norm=False):
    return mt_config(E, H, A, V, int(layer_norm), int(tied_output), k_max,
                     MT_BF16 if gemm == "bf16" else MT_F32, ln_eps, transitions, src_V, int(dual_source),
                     enc_transitions, int(enc_layer_norm))


class Model:
    """Owns an mt_model handle (freed with mt_free)."""

    def __init__(self, handle: int, cfg: mt_config):
        self.handle = handle
        self.cfg = cfg

    def __del__(self):
        if getattr(self, "handle", None):
            try:
                lib().mt_free(self.handle)
            except Exception:
                pass
            self.handle = None


def mt_load_weights(cfg: mt_config, weights: Dict[str, np.ndarray]) -> Model:
    """weights: host fp32 arrays by field name (see mt_weights)."""
    keep = {}
    w = mt_weights()
    for n in WEIGHT_FIELDS:
        a = weights.get(n)
        if a is None:
            continue
        a = np.ascontiguousarray(a, dtype=np.float32)
        keep[n] = a
        setattr(w, n, a.ctypes.data_as(_fp))
    h = _vp()
    _check(lib().mt_load_weights(C.byref(cfg), C.byref(w), C.byref(h)))
    return Model(h.value, cfg)


def mt_ensemble_logp(model: Model, logps, weights, M: int, out, stream=None):
    """out = sum_i weights[i] * logps[i] over [M, V] (device tensors; out may be one of them)."""
    n = len(logps)
    ptrs = (_vp * n)(*[_ptr(x) for x in logps])
    w = (C.c_float * n)(*[float(x) for x in weights])
    _check(lib().mt_ensemble_logp(model.handle, n, ptrs, w, M, _ptr(out), _stream(stream)))


def mt_beam_finish(model: Model, B, K, step, eos, alpha, final, tok, bp, row, score, beam, fin_count, hist_tok,
                   hist_bp, fin_score, fin_norm, fin_step, fin_parent, fin_tok, stream=None):
    _check(lib().mt_beam_finish(model.handle, B, K, step, eos, alpha, int(bool(final)),
                                *[_ptr(x) for x in (tok, bp, row, score, beam, fin_count, hist_tok, hist_bp,
                                                    fin_score, fin_norm, fin_step, fin_parent, fin_tok)],
                                _stream(stream)))


def mt_encode_workspace_bytes(model: Model, B: int, S: int) -> int:
    return int(lib().mt_encode_workspace_bytes(model.handle, B, S))


def mt_encode(model: Model, B, S, src_tok, mask, ctx_out, ws, ws_bytes=None, stream=None):
    ws_bytes = ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes
    _check(lib().mt_encode(model.handle, B, S, _ptr(src_tok), _ptr(mask), _ptr(ctx_out), _ptr(ws), ws_bytes,
                           _stream(stream)))


def mt_free(model: Model):
    if model.handle:
        _check(lib().mt_free(model.handle))
        model.handle = None


def mt_workspace_bytes(model: Model, B: int, K: int, S: int) -> int:
    return int(lib().mt_workspace_bytes(model.handle, B, K, S))


def mt_precompute_ctx(model: Model, B, S, ctx, mask, pctx_out, s0_out, ws, ws_bytes=None, stream=None):
    ws_bytes = ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes
    _check(lib().mt_precompute_ctx(model.handle, B, S, _ptr(ctx), _ptr(mask), _ptr(pctx_out), _ptr(s0_out),
                                   _ptr(ws), ws_bytes, _stream(stream)))


def mt_precompute_ctx_noalloc(model: Model, B, S, ctx, mask, pctx_out, s0_out, stream=None):
    _check(lib().mt_precompute_ctx_noalloc(model.handle, B, S, _ptr(ctx), _ptr(mask), _ptr(pctx_out), _ptr(s0_out),
                                           _stream(stream)))


def mt_decoder_step(model: Model, B, K, S, prev_tok, src_row, n_state_rows, state_in, ctx, pctx, mask,
                    state_out, logp_out=None, attn_out=None, taps=None, ws=None, ws_bytes=None, stream=None):
    ws_bytes = ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes
    tp = None
    if taps:
        tp = mt_taps(_ptr(taps.get("s1")), _ptr(taps.get("c")), _ptr(taps.get("t")))
    _check(lib().mt_decoder_step(model.handle, B, K, S, _ptr(prev_tok), _ptr(src_row), n_state_rows,
                                 _ptr(state_in), _ptr(ctx), _ptr(pctx), _ptr(mask), _ptr(state_out),
                                 _ptr(logp_out), _ptr(attn_out), C.byref(tp) if tp is not None else None,
                                 _ptr(ws), ws_bytes, _stream(stream)))


def mt_decoder_step_dual(model: Model, B, K, S, prev_tok, src_row, n_state_rows, state_in, ctx, pctx, mask, S2,
                         ctx2, pctx2, mask2, state_out, logp_out=None, attn_out=None, taps=None, ws=None,
                         ws_bytes=None, stream=None):
    ws_bytes = ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes
    tp = None
    if taps:
        tp = mt_taps(_ptr(taps.get("s1")), _ptr(taps.get("c")), _ptr(taps.get("t")))
    _check(lib().mt_decoder_step_dual(model.handle, B, K, S, _ptr(prev_tok), _ptr(src_row), n_state_rows,
                                      _ptr(state_in), _ptr(ctx), _ptr(pctx), _ptr(mask), S2, _ptr(ctx2), _ptr(pctx2),
                                      _ptr(mask2), _ptr(state_out), _ptr(logp_out), _ptr(attn_out),
                                      C.byref(tp) if tp is not None else None, _ptr(ws), ws_bytes, _stream(stream)))


def mt_precompute_keys2(model: Model, B, S2, ctx2, mask2, pctx2_out, ws, ws_bytes=None, stream=None):
    ws_bytes = ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes
    _check(lib().mt_precompute_keys2(model.handle, B, S2, _ptr(ctx2), _ptr(mask2), _ptr(pctx2_out), _ptr(ws),
                                     ws_bytes, _stream(stream)))


def mt_beam_topk(model: Model, B, K, prev_score, logp, score_out, tok_out, bp_out, row_out=None, ws=None,
                 ws_bytes=None, stream=None):
    ws_bytes = ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes
    _check(lib().mt_beam_topk(model.handle, B, K, _ptr(prev_score), _ptr(logp), _ptr(score_out), _ptr(tok_out),
                              _ptr(bp_out), _ptr(row_out), _ptr(ws), ws_bytes, _stream(stream)))


def mt_device_errors(model: Model) -> int:
    f = C.c_int32(0)
    _check(lib().mt_device_errors(model.handle, C.byref(f)))
    return int(f.value)


def mt_ensemble_step(model: Model, member, n_members, weight, B, K, S, prev_tok, src_row, n_state_rows, state_in, ctx,
                     pctx, mask, state_out, comb_logits, ws, ws_bytes=None, stream=None):
    ws_bytes = ws.numel() * ws.element_size() if ws_bytes is None else ws_bytes
    _check(lib().mt_ensemble_step(model.handle, member, n_members, float(weight), B, K, S, _ptr(prev_tok), _ptr(src_row),
                                  n_state_rows, _ptr(state_in), _ptr(ctx), _ptr(pctx), _ptr(mask), _ptr(state_out),
                                  _ptr(comb_logits), _ptr(ws), ws_bytes, _stream(stream)))


def mt_beam_nbest(model: Model, B, K, steps, hist_tok, hist_bp, fin_count, fin_norm, fin_step, fin_parent, fin_tok,
                  order, seq, stream=None):
    ld_seq = seq.shape[1]
    _check(lib().mt_beam_nbest(model.handle, B, K, steps, _ptr(hist_tok), _ptr(hist_bp), _ptr(fin_count),
                               _ptr(fin_norm), _ptr(fin_step), _ptr(fin_parent), _ptr(fin_tok), _ptr(order), _ptr(seq),
                               ld_seq, _stream(stream)))


def mt_set_state_reuse(model: Model, on: bool):
    _check(lib().mt_set_state_reuse(model.handle, 1 if on else 0))


def mt_ensemble_joint_ok(models) -> bool:
    n = len(models)
    hs = (_vp * n)(*[m.handle for m in models])
    return bool(lib().mt_ensemble_joint_ok(n, hs))


def mt_ensemble_topk(models, weights, wss, B, K, prev_score, comb_logits, score_out, tok_out, bp_out, row_out=None,
                     row_const_out=None, stream=None):
    n = len(models)
    hs = (_vp * n)(*[m.handle for m in models])
    ws_ = (C.c_float * n)(*[float(x) for x in weights])
    wp = (_vp * n)(*[_ptr(w) for w in wss])
    wb = (C.c_size_t * n)(*[w.numel() * w.element_size() for w in wss])
    _check(lib().mt_ensemble_topk(n, hs, ws_, wp, wb, B, K, _ptr(prev_score), _ptr(comb_logits), _ptr(score_out),
                                  _ptr(tok_out), _ptr(bp_out), _ptr(row_out), _ptr(row_const_out), _stream(stream)))


def mt_recomputed_rows(model: Model) -> int:
    n = C.c_int64(0)
    _check(lib().mt_recomputed_rows(model.handle, C.byref(n)))
    return int(n.value)


def mt_profile_enable(model: Model, kernels=("VOCAB_GEMM",)):
    """Times the given kernel classes (names or ids) with HIP events; () turns timing off."""
    mask = 0
    for k in kernels:
        mask |= 1 << (KERNEL_ID[k] if isinstance(k, str) else int(k))
    _check(lib().mt_profile_enable(model.handle, mask))


def mt_profile_sample(model: Model, every: int):
    """Times one launch in `every` of each selected class."""
    _check(lib().mt_profile_sample(model.handle, int(every)))


def mt_profile_reset(model: Model):
    _check(lib().mt_profile_reset(model.handle))


def mt_profile_query(model: Model, kernel) -> tuple:
    k = KERNEL_ID[kernel] if isinstance(kernel, str) else int(kernel)
    ms, n = C.c_double(0), C.c_int64(0)
    _check(lib().mt_profile_query(model.handle, k, C.byref(ms), C.byref(n)))
    return float(ms.value), int(n.value)


# ---- recurrent layer: products in 8 bits, causal convolution, selective scan ----------------------
#
# Row matrices are torch tensors [..., width] whose last dimension is contiguous and whose rows are
# equally spaced (a column range of a wider matrix is fine); sizes come from their shapes.

class I8Matrix:
    """Owns an mt_i8_matrix handle (freed with mt_i8_free)."""

    def __init__(self, handle: int, K: int, N: int, device):
        self.handle, self.K, self.N, self.device = handle, K, N, device

    def __del__(self):
        if getattr(self, "handle", None):
            try:
                lib().mt_i8_free(self.handle)
            except Exception:
                pass
            self.handle = None


class Ssm:
    """Owns an mt_ssm handle (freed with mt_ssm_free)."""

    def __init__(self, handle: int, cfg: mt_ssm_config, device):
        import torch
        self.handle, self.cfg, self.device = handle, cfg, device
        self.D, self.W, self.N, self.GN = cfg.D, cfg.W, cfg.N, cfg.G * cfg.N
        self.dtype = torch.bfloat16 if cfg.dtype == MT_BF16 else torch.float32
        self.f32, self.i32 = torch.float32, torch.int32

    def __del__(self):
        if getattr(self, "handle", None):
            try:
                lib().mt_ssm_free(self.handle)
            except Exception:
                pass
            self.handle = None


def _current_device():
    import torch
    return torch.device("cuda", torch.cuda.current_device()) if torch.cuda.is_available() else None


def _bad(t, name, shape, dtype, device):
    return ValueError(f"{name}: need a {dtype} tensor of shape {tuple(shape)} on {device}, got {t.dtype} "
                      f"{tuple(t.shape)} on {t.device}")


def _rows(t, name, shape, dtype, device):
    """(address, row stride) of a row matrix of two or three dimensions."""
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        raise _bad(t, name, shape, dtype, device)
    st, width = t.stride(), shape[-1]
    if st[-1] != 1 and width > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    if len(st) == 2:
        return t.data_ptr(), st[0] if shape[0] > 1 else width
    B, S = shape[0], shape[1]
    ld = st[1] if S > 1 else (st[0] if B > 1 else width)
    if B > 1 and st[0] != S * ld:
        raise ValueError(f"the rows of {name} must be equally spaced")
    return t.data_ptr(), ld


def _packed(t, name, shape, dtype, device):
    """Address of a contiguous tensor of a given shape, or None."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or t.device != device or not t.is_contiguous():
        raise _bad(t, name + " (contiguous)", shape, dtype, device)
    return t.data_ptr()


def _space(ws, device):
    """(address, bytes) of a workspace."""
    if ws.device != device or not ws.is_contiguous():
        raise ValueError(f"ws: need a contiguous tensor on {device}")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _host_or_device(a):
    """An fp32 array and its address: a device tensor stays where it is.  What another device than the current one
    still does for it is waited for: the load waits for its own only."""
    import torch
    if isinstance(a, torch.Tensor):
        a = a.detach().to(torch.float32).contiguous()
        if a.is_cuda and a.device != _current_device():
            torch.cuda.synchronize(a.device)
        return a, a.data_ptr()
    a = np.ascontiguousarray(a, np.float32)
    return a, a.ctypes.data


def mt_i8_load(W, bias=None) -> I8Matrix:
    """W [K, N], bias [N] (or None): fp32, numpy arrays or torch tensors on any device."""
    if len(W.shape) != 2 or (bias is not None and tuple(bias.shape) != (W.shape[1],)):
        raise ValueError("need W [K, N] and bias [N]")
    K, N = (int(n) for n in W.shape)
    w, wp = _host_or_device(W)
    b, bp = _host_or_device(bias) if bias is not None else (None, None)
    h = _vp()
    _check(lib().mt_i8_load(K, N, wp, bp, C.byref(h)))
    return I8Matrix(h.value, K, N, _current_device())


def mt_i8_free(mat: I8Matrix):
    if mat.handle:
        _check(lib().mt_i8_free(mat.handle))
        mat.handle = None


def mt_i8_workspace_bytes(mat: I8Matrix, M: int) -> int:
    return int(lib().mt_i8_workspace_bytes(mat.handle, M))


def _io(t, name):
    import torch
    if t.dtype == torch.float32:
        return MT_F32
    if t.dtype == torch.bfloat16:
        return MT_BF16
    raise ValueError(f"{name} is {t.dtype}: need float32 or bfloat16")


def mt_i8_product(mat: I8Matrix, x, y, ws, stream=None):
    """y = x W + bias with both operands in 8 bits; x [..., K], y [..., N] of the same leading shape."""
    lead, dev = x.shape[:-1], mat.device
    if len(lead) != 1 and len(lead) != 2:
        raise ValueError("x must have two or three dimensions")
    xt, yt = _io(x, "x"), _io(y, "y")
    xp, ldx = _rows(x, "x", lead + (mat.K,), x.dtype, dev)
    yp, ldy = _rows(y, "y", lead + (mat.N,), y.dtype, dev)
    _check(lib().mt_i8_product(mat.handle, lead.numel(), xp, xt, ldx, yp, yt, ldy, *_space(ws, dev), _stream_on(stream, dev)))


def make_ssm_config(D, N, *, groups=1, conv=0, conv_silu=True, dtype="f32"):
    return mt_ssm_config(D, N, groups, conv, MT_BF16 if dtype == "bf16" else MT_F32, int(conv_silu))


def mt_ssm_load(cfg: mt_ssm_config, weights) -> Ssm:
    """weights: fp32 numpy arrays or torch tensors by field name (see mt_ssm_weights)."""
    shapes = dict(A=(cfg.D, cfg.N), dt_bias=(cfg.D,), skip=(cfg.D,), conv_w=(cfg.D, cfg.W), conv_b=(cfg.D,))
    w, keep = mt_ssm_weights(), []
    for n in SSM_WEIGHT_FIELDS:
        a = weights.get(n)
        if a is None:
            continue
        if hasattr(a, "detach"):
            a = a.detach().float().cpu().numpy()
        a = np.ascontiguousarray(a, np.float32)
        if a.shape != shapes[n]:
            raise ValueError(f"{n} has shape {a.shape}: need {shapes[n]}")
        keep.append(a)
        setattr(w, n, a.ctypes.data_as(_fp))
    h = _vp()
    _check(lib().mt_ssm_load(C.byref(cfg), C.byref(w), C.byref(h)))
    return Ssm(h.value, mt_ssm_config.from_buffer_copy(cfg), _current_device())


def mt_ssm_free(cell: Ssm):
    if cell.handle:
        _check(lib().mt_ssm_free(cell.handle))
        cell.handle = None


def mt_ssm_workspace_bytes(cell: Ssm, B: int, S: int) -> int:
    return int(lib().mt_ssm_workspace_bytes(cell.handle, B, S))


def mt_ssm_device_errors(cell: Ssm) -> int:
    f = C.c_int32(0)
    _check(lib().mt_ssm_device_errors(cell.handle, C.byref(f)))
    return int(f.value)


def mt_ssm_conv(cell: Ssm, x, y, *, lens=None, state_in=None, state_out=None, stream=None):
    """x, y [B, S, D]; lens [B] int32; state_in, state_out [B, W-1, D]."""
    dt, dev, D = cell.dtype, cell.device, cell.D
    B, S = x.shape[:-1]
    st, rows = (B, max(cell.W - 1, 0), D), (B, S, D)
    xp, ldx = _rows(x, "x", rows, dt, dev)
    yp, ldy = _rows(y, "y", rows, dt, dev)
    _check(lib().mt_ssm_conv(cell.handle, B, S, _packed(lens, "lens", (B,), cell.i32, dev), xp, ldx,
                             _packed(state_in, "state_in", st, dt, dev), yp, ldy,
                             _packed(state_out, "state_out", st, dt, dev), _stream_on(stream, dev)))


def mt_ssm_conv_step(cell: Ssm, x, y, state_in, state_out, *, src_row=None, stream=None):
    """x, y [M, D]; state_in [rows, W-1, D], state_out [M, W-1, D]; src_row [M] int32."""
    dt, dev, D, W1 = cell.dtype, cell.device, cell.D, max(cell.W - 1, 0)
    M, = x.shape[:-1]
    n, rows = state_in.shape[0] if state_in is not None else M, (M, D)
    xp, ldx = _rows(x, "x", rows, dt, dev)
    yp, ldy = _rows(y, "y", rows, dt, dev)
    _check(lib().mt_ssm_conv_step(cell.handle, M, _packed(src_row, "src_row", (M,), cell.i32, dev), n, xp, ldx,
                                  _packed(state_in, "state_in", (n, W1, D), dt, dev), yp, ldy,
                                  _packed(state_out, "state_out", (M, W1, D), dt, dev), _stream_on(stream, dev)))


def _scan_rows(cell, lead, x, dt, bmat, cmat, y, z):
    """The row-matrix arguments of the scan in the order of the C calls, without the states."""
    t, dev = cell.dtype, cell.device
    rows, bc = lead + (cell.D,), lead + (cell.GN,)
    xp, ldx = _rows(x, "x", rows, t, dev)
    dp, ldd = _rows(dt, "dt", rows, t, dev)
    bp, ldb = _rows(bmat, "bmat", bc, t, dev)
    cp, ldc = _rows(cmat, "cmat", bc, t, dev)
    if ldb != ldc:
        raise ValueError("bmat and cmat must have the same row stride")
    zp, ldz = _rows(z, "z", rows, t, dev) if z is not None else (None, 0)
    yp, ldy = _rows(y, "y", rows, t, dev)
    return xp, ldx, dp, ldd, bp, cp, ldb, zp, ldz, yp, ldy


def mt_ssm_scan(cell: Ssm, x, dt, bmat, cmat, y, *, z=None, lens=None, state_in=None, state_out=None, ws, stream=None):
    """x, dt, z, y [B, S, D]; bmat, cmat [B, S, G*N]; lens [B] int32; state_in, state_out [B, D, N] fp32."""
    dev = cell.device
    B, S = lead = x.shape[:-1]
    r = _scan_rows(cell, lead, x, dt, bmat, cmat, y, z)
    st = (B, cell.D, cell.N)
    _check(lib().mt_ssm_scan(cell.handle, B, S, _packed(lens, "lens", (B,), cell.i32, dev), *r[:9],
                             _packed(state_in, "state_in", st, cell.f32, dev), r[9], r[10],
                             _packed(state_out, "state_out", st, cell.f32, dev), *_space(ws, dev), _stream_on(stream, dev)))


def mt_ssm_step(cell: Ssm, x, dt, bmat, cmat, y, state_in, state_out, *, z=None, src_row=None, stream=None):
    """x, dt, z, y [M, D]; bmat, cmat [M, G*N]; state_in [rows, D, N], state_out [M, D, N] fp32; src_row [M] int32."""
    dev = cell.device
    M, = lead = x.shape[:-1]
    n = state_in.shape[0]
    r = _scan_rows(cell, lead, x, dt, bmat, cmat, y, z)
    _check(lib().mt_ssm_step(cell.handle, M, _packed(src_row, "src_row", (M,), cell.i32, dev), n, *r[:9],
                             _packed(state_in, "state_in", (n, cell.D, cell.N), cell.f32, dev), r[9], r[10],
                             _packed(state_out, "state_out", (M, cell.D, cell.N), cell.f32, dev), _stream_on(stream, dev)))
