"""Thin ctypes binding of libflashloop.so (argument marshalling only).

Every function takes torch tensors that live on the ROCm device, checks dtype/shape/contiguity,
allocates outputs with torch, and passes raw device pointers plus the current HIP stream to the C ABI
declared in include/flashloop.h.  All arithmetic happens in the library's HIP kernels; if the library
is missing this module raises instead of falling back to anything else.
"""
from __future__ import annotations

import ctypes
import math
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libflashloop.so")

AXIS_TOKEN = 0
AXIS_CHANNEL = 1
DQ_COMPACT = 0
DQ_COMMIT = 1
ATTN_DENSE = 1
PASS_ADD, PASS_SUBTRACT, PASS_BOTH = 0, 1, 2
ROPE_SCALING = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}
ROPE_LAYOUT = {"half": 0, "interleaved": 1}

_c_p = ctypes.c_void_p
_c_i = ctypes.c_int
_c_d = ctypes.c_double
_c_f = ctypes.c_float
_c_sz = ctypes.c_size_t
_c_l = ctypes.c_int64

_SIGNATURES = {
    "fl_status_str": (ctypes.c_char_p, [_c_i]),
    "fl_last_error": (ctypes.c_char_p, []),
    "fl_abi_version": (_c_i, []),
    "fl_set_index_checks": (None, [_c_i]),
    "fl_index_checks": (_c_i, []),
    "fl_select_tokens": (_c_i, [_c_p, _c_p, _c_p, _c_p, _c_i, _c_i, _c_i, _c_p, _c_i, _c_i, _c_i, _c_d,
                                _c_p, _c_p, _c_p, _c_p]),
    "fl_kv_residual_quant": (_c_i, [_c_p, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i,
                                    _c_p, _c_p, _c_p, _c_p, _c_p]),
    "fl_kv_residual_quant_commit": (_c_i, [_c_p, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i,
                                           _c_p, _c_p, _c_p, _c_p]),
    "fl_kv_residual_dequant": (_c_i, [_c_p, _c_p, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i,
                                      _c_i, _c_i, _c_p, _c_p, _c_p]),
    "fl_kv_residual_dequant_kv": (_c_i, [_c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i,
                                         _c_i, _c_i, _c_i, _c_p, _c_p, _c_p, _c_p, _c_p]),
    "fl_kv_residual_quant_kv": (_c_i, [_c_p, _c_p, _c_p, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i,
                                       _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_i, _c_p]),
    "fl_kv_residual_quant_kv_v16": (_c_i, [_c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i,
                                           _c_i, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p]),
    "fl_kv_f16_rows": (_c_i, [_c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i, _c_p, _c_p]),
    "fl_loop_sparse_attn_ws": (_c_sz, [_c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i]),
    "fl_loop_sparse_attn": (_c_i, [_c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_i, _c_p, _c_i, _c_i,
                                   _c_i, _c_i, _c_i, _c_i, _c_f, _c_i, _c_p, _c_p, _c_p, _c_sz, _c_p]),
    "fl_loop_sparse_attn_terms": (_c_i, [_c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p, _c_i, _c_p, _c_i, _c_i,
                                         _c_i, _c_i, _c_i, _c_i, _c_f, _c_p, _c_p, _c_p, _c_p, _c_p, _c_i, _c_p,
                                         _c_p, _c_p, _c_sz, _c_p]),
    "fl_loop_subtract_terms_supported": (_c_i, [_c_i, _c_i, _c_i, _c_i, _c_i]),
    "fl_attn_kernel_name": (ctypes.c_char_p, [_c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i]),
    "fl_loop_subtract_terms": (_c_i, [_c_p, _c_p, _c_p, _c_p, _c_i, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_f,
                                      _c_p, _c_p, _c_p, _c_p]),
    "fl_loop_sparse_attn_terms_v16": (_c_i, [_c_p, _c_p, _c_p, _c_p, _c_p, _c_i, _c_p, _c_i, _c_i, _c_i, _c_i,
                                             _c_i, _c_i, _c_f, _c_p, _c_p, _c_p, _c_p, _c_p, _c_i, _c_p, _c_p,
                                             _c_p]),
    "fl_loop_subtract_terms_v16": (_c_i, [_c_p, _c_p, _c_p, _c_p, _c_p, _c_i, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i,
                                          _c_i, _c_f, _c_p, _c_p, _c_p, _c_p]),
    "fl_column_scores_ws": (_c_sz, [_c_i, _c_i, _c_i]),
    "fl_column_scores": (_c_i, [_c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_p, _c_p, _c_sz, _c_p]),
    "fl_select_columns": (_c_i, [_c_p, _c_i, _c_i, _c_i, _c_i, _c_i, _c_p, _c_p]),
    "fl_decode_step_ws": (_c_sz, [_c_i, _c_i, _c_i, _c_i, _c_i, _c_i]),
    "fl_decode_step": (_c_i, [_c_p, _c_p, _c_p, _c_p, _c_i, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_f, _c_p, _c_p,
                              _c_i, _c_i, _c_i, _c_p, _c_p, _c_p, _c_p, _c_sz, _c_p]),
    "fl_decode_step_noalloc": (_c_i, [_c_p, _c_p, _c_p, _c_p, _c_i, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_f, _c_p,
                                      _c_p, _c_i, _c_i, _c_i, _c_p, _c_p, _c_p, _c_p]),
    "fl_prune_columns_ws": (_c_sz, [_c_i, _c_i, _c_i, _c_i, _c_i]),
    "fl_kv_keep_recent": (_c_i, [_c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_p, _c_p, _c_p]),
    "fl_prune_columns": (_c_i, [_c_p, _c_p, _c_p, _c_i, _c_p, _c_i, _c_p, _c_i, _c_i, _c_i, _c_i, _c_d, _c_i, _c_i,
                                _c_p, _c_p, _c_p, _c_sz, _c_p]),
    "fl_rope_table": (_c_i, [_c_i, _c_i, _c_d, _c_i, _c_d, _c_d, _c_d, _c_d, _c_p, _c_p]),
    "fl_rope": (_c_i, [_c_p, _c_l, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_p, _c_l, _c_p]),
    "fl_paged_append": (_c_i, [_c_p, _c_l, _c_p, _c_l, _c_i, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_p, _c_i, _c_i, _c_i,
                               _c_p, _c_i, _c_i, _c_i, _c_i, _c_p, _c_p, _c_p, _c_p, _c_p]),
    "fl_paged_attn_ws": (_c_sz, [_c_i] * 11),
    "fl_paged_attn": (_c_i, [_c_p, _c_l, _c_i, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i, _c_p, _c_i, _c_i, _c_i, _c_p,
                             _c_i, _c_i, _c_i, _c_i, _c_p, _c_p, _c_p, _c_p, _c_f, _c_i, _c_i, _c_i, _c_i, _c_p, _c_l,
                             _c_p, _c_p, _c_sz, _c_p]),
    "fl_packed_attn_ws": (_c_sz, [_c_i] * 9),
    "fl_packed_attn": (_c_i, [_c_p, _c_l, _c_p, _c_l, _c_p, _c_l, _c_i, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i, _c_i, _c_p,
                              _c_i, _c_i, _c_i, _c_f, _c_i, _c_i, _c_i, _c_p, _c_l, _c_p, _c_p, _c_sz, _c_p]),
    "fl_paged4_append": (_c_i, [_c_p, _c_l, _c_p, _c_l, _c_i, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_p, _c_i, _c_i, _c_i,
                                _c_p, _c_i, _c_i, _c_i, _c_i, _c_p, _c_p, _c_p, _c_p, _c_p, _c_l, _c_p, _c_l, _c_p]),
    "fl_paged4_read": (_c_i, [_c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_p, _c_i, _c_i, _c_i, _c_i, _c_p, _c_p, _c_p, _c_p, _c_i,
                              _c_p, _c_l, _c_p, _c_l, _c_p]),
    "fl_paged4_attn_ws": (_c_sz, [_c_i] * 11),
    "fl_paged4_attn": (_c_i, [_c_p, _c_l, _c_i, _c_p, _c_p, _c_i, _c_i, _c_i, _c_i, _c_i, _c_p, _c_i, _c_i, _c_i, _c_p,
                              _c_i, _c_i, _c_i, _c_i, _c_p, _c_p, _c_p, _c_p, _c_f, _c_i, _c_i, _c_i, _c_i, _c_p, _c_l,
                              _c_p, _c_p, _c_sz, _c_p]),
}

EXPORTS = tuple(_SIGNATURES)

_lib = None


class FlashLoopError(RuntimeError):
    pass


def load(path: str = LIB_PATH):
    """Load the HIP library (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise FlashLoopError(f"{path} is missing: build it with `python -m paper_2609_29812_amd.build`")
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def set_index_checks(on: bool):
    """Turn the library's index-list checks on or off (every call then validates its lists on the host)."""
    load().fl_set_index_checks(1 if on else 0)


def index_checks() -> bool:
    """Whether the library's index-list checks are on."""
    return load().fl_index_checks() != 0


def _check(rc: int, fn: str):
    if rc != 0:
        lib = load()
        raise FlashLoopError(f"{fn}: {lib.fl_status_str(rc).decode()}: {lib.fl_last_error().decode()}")


# The calls below run on the host between launches of a few microseconds each, so the marshalling is kept short:
# pointers as plain integers (c_void_p arguments take them), the stream by one C call instead of the Stream object
# (5 us of a call's 16), and a tensor that passes its checks passes them in one expression.
def _p(t):
    return None if t is None else t.data_ptr()


# (the C call is private to torch; without it the public form)
if hasattr(torch._C, "_cuda_getCurrentRawStream") and hasattr(torch._C, "_cuda_getDevice"):
    def _stream():
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
else:
    def _stream():
        return torch.cuda.current_stream().cuda_stream


def _dev(t, dtype, name, shape=None):
    if t is None or (t.dtype is dtype and t.is_cuda and t.is_contiguous() and (shape is None or t.shape == shape)):
        return
    if not t.is_cuda:
        raise FlashLoopError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise FlashLoopError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise FlashLoopError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise FlashLoopError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


# ---- (1) token selection ----------------------------------------------------------------------------
def select_tokens(k_cur, k_prev, v_cur, v_prev, k, cand=None, normalize=True, eps=1e-6, slot=True,
                  out_key=None, out_idx=None, out_slot=None):
    """Active rows of the loop: returns (idx int32 [B, k], slot int32 [B, N] or None, key fp32 [B, n])."""
    shape = k_cur.shape
    B, N = shape[:2]
    D = k_cur.numel() // (B * N)
    for name, t in (("k_cur", k_cur), ("k_prev", k_prev), ("v_cur", v_cur), ("v_prev", v_prev)):
        _dev(t, torch.bfloat16, name, shape)
    n_cand = N if cand is None else cand.shape[1]
    _dev(cand, torch.int32, "cand", None if cand is None else (B, n_cand))
    dev = k_cur.device
    out_key = torch.empty(B, n_cand, dtype=torch.float32, device=dev) if out_key is None else out_key
    out_idx = torch.empty(B, k, dtype=torch.int32, device=dev) if out_idx is None else out_idx
    if slot and out_slot is None:
        out_slot = torch.empty(B, N, dtype=torch.int32, device=dev)
    rc = load().fl_select_tokens(_p(k_cur), _p(k_prev), _p(v_cur), _p(v_prev), B, N, D, _p(cand), n_cand,
                                 k, 1 if normalize else 0, eps, _p(out_key), _p(out_idx),
                                 _p(out_slot) if slot else None, _stream())
    _check(rc, "fl_select_tokens")
    return out_idx, (out_slot if slot else None), out_key


# ---- (2) residual codec -----------------------------------------------------------------------------
def meta_shape(B, k, H, d, group, axis):
    return (B, -(-k // group), H, d) if axis == AXIS_TOKEN else (B, k, H, d // group)


def kv_residual_quant(x_cur, x_ref, idx, bits, group, axis, rows=True, out=None):
    """Quantize the residual of rows idx (None = all rows).  Returns (codes, scale, zero, rows)."""
    B, N, H, d = x_cur.shape
    _dev(x_cur, torch.bfloat16, "x_cur")
    _dev(x_ref, torch.bfloat16, "x_ref", x_cur.shape)
    k = N if idx is None else idx.shape[1]
    _dev(idx, torch.int32, "idx", None if idx is None else (B, k))
    dev = x_cur.device
    o = out or {}
    codes = o.get("codes")
    if codes is None:
        codes = torch.empty(B, k, H, d * bits // 8, dtype=torch.uint8, device=dev)
    scale = zero = None
    if bits != 16:
        shp = meta_shape(B, k, H, d, group, axis)
        scale = o.get("scale") if o.get("scale") is not None else torch.empty(shp, dtype=torch.float16, device=dev)
        zero = o.get("zero") if o.get("zero") is not None else torch.empty(shp, dtype=torch.float16, device=dev)
    out_rows = None
    if rows is True:
        out_rows = torch.empty(B, k, H, d, dtype=torch.bfloat16, device=dev)
    elif rows is not None and rows is not False:
        out_rows = rows
    rc = load().fl_kv_residual_quant(_p(x_cur), _p(x_ref), _p(idx), k, B, N, H, d, bits, group, axis,
                                     _p(codes), _p(scale), _p(zero), _p(out_rows), _stream())
    _check(rc, "fl_kv_residual_quant")
    return codes, scale, zero, out_rows


def kv_residual_quant_commit(x_cur, x_hat, idx, bits, group, axis, out=None):
    """Quantize the residual of rows idx against x_hat and commit the reconstruction into x_hat in place.
    Returns (codes, scale, zero)."""
    B, N, H, d = x_cur.shape
    _dev(x_cur, torch.bfloat16, "x_cur")
    _dev(x_hat, torch.bfloat16, "x_hat", x_cur.shape)
    k = N if idx is None else idx.shape[1]
    _dev(idx, torch.int32, "idx", None if idx is None else (B, k))
    dev = x_cur.device
    o = out or {}
    codes = o.get("codes")
    if codes is None:
        codes = torch.empty(B, k, H, d * bits // 8, dtype=torch.uint8, device=dev)
    scale = zero = None
    if bits != 16:
        shp = meta_shape(B, k, H, d, group, axis)
        scale = o.get("scale") if o.get("scale") is not None else torch.empty(shp, dtype=torch.float16, device=dev)
        zero = o.get("zero") if o.get("zero") is not None else torch.empty(shp, dtype=torch.float16, device=dev)
    rc = load().fl_kv_residual_quant_commit(_p(x_cur), _p(x_hat), _p(idx), k, B, N, H, d, bits, group, axis,
                                            _p(codes), _p(scale), _p(zero), _stream())
    _check(rc, "fl_kv_residual_quant_commit")
    return codes, scale, zero


def kv_residual_quant_kv(k_cur, k_ref, v_cur, v_ref, idx, bits, group, mode=DQ_COMPACT, rows=True, v_f16=None):
    """Keys (token axis) and values (channel axis) in one call.  COMPACT: returns
    ((codes, scale, zero, rows) for keys, the same for values), rows None unless rows=True;
    COMMIT: rows idx of k_ref / v_ref are updated in place and the rows entries are None; with v_f16 (fp16
    [B, N, H, d], COMMIT only) its rows idx receive the fp16 copy of the updated values
    (fl_kv_residual_quant_kv_v16)."""
    B, N, H, d = shape = k_cur.shape
    _dev(k_cur, torch.bfloat16, "k_cur")
    _dev(v_cur, torch.bfloat16, "v_cur", shape)
    _dev(k_ref, torch.bfloat16, "k_ref", shape)
    _dev(v_ref, torch.bfloat16, "v_ref", shape)
    k = N if idx is None else idx.shape[1]
    _dev(idx, torch.int32, "idx", None if idx is None else (B, k))
    dev = k_cur.device

    def outputs(axis):
        codes = torch.empty(B, k, H, d * bits // 8, dtype=torch.uint8, device=dev)
        scale = zero = None
        if bits != 16:
            shp = meta_shape(B, k, H, d, group, axis)
            scale = torch.empty(*shp, dtype=torch.float16, device=dev)
            zero = torch.empty_like(scale)
        out_rows = None
        if mode == DQ_COMPACT and rows:
            out_rows = torch.empty(B, k, H, d, dtype=torch.bfloat16, device=dev)
        return codes, scale, zero, out_rows

    ko, vo = outputs(AXIS_TOKEN), outputs(AXIS_CHANNEL)
    if v_f16 is not None:
        if mode != DQ_COMMIT:
            raise FlashLoopError("kv_residual_quant_kv: v_f16 needs mode=DQ_COMMIT")
        _dev(v_f16, torch.float16, "v_f16", k_cur.shape)
        rc = load().fl_kv_residual_quant_kv_v16(_p(k_cur), _p(k_ref), _p(v_cur), _p(v_ref), _p(v_f16), _p(idx), k,
                                                B, N, H, d, bits, group, _p(ko[0]), _p(ko[1]), _p(ko[2]),
                                                _p(vo[0]), _p(vo[1]), _p(vo[2]), _stream())
        _check(rc, "fl_kv_residual_quant_kv_v16")
        return ko, vo
    rc = load().fl_kv_residual_quant_kv(_p(k_cur), _p(k_ref), _p(v_cur), _p(v_ref), _p(idx), k, B, N, H, d, bits,
                                        group, _p(ko[0]), _p(ko[1]), _p(ko[2]), _p(vo[0]), _p(vo[1]), _p(vo[2]),
                                        _p(ko[3]), _p(vo[3]), mode, _stream())
    _check(rc, "fl_kv_residual_quant_kv")
    return ko, vo


def kv_f16_rows(x, idx=None, out=None):
    """fp16 copy of rows of a bf16 [B, N, H, d] tensor (fl_kv_f16_rows): every row when idx is None, else
    rows idx of `out` (fp16 [B, N, H, d], allocated when None); returns out."""
    B, N, H, d = x.shape
    _dev(x, torch.bfloat16, "x")
    k = N if idx is None else idx.shape[1]
    _dev(idx, torch.int32, "idx", None if idx is None else (B, k))
    out = torch.empty(B, N, H, d, dtype=torch.float16, device=x.device) if out is None else out
    _dev(out, torch.float16, "out", x.shape)
    rc = load().fl_kv_f16_rows(_p(x), _p(idx), k, B, N, H, d, _p(out), _stream())
    _check(rc, "fl_kv_f16_rows")
    return out


def kv_residual_dequant_kv(k_enc, v_enc, idx, bits, group, k_hat, v_hat, mode=DQ_COMPACT):
    """Keys (token axis) and values (channel axis) in one call; k_enc / v_enc = (codes, scale, zero).
    COMPACT: returns (key rows, value rows) [B, k, H, d]; COMMIT: updates k_hat and v_hat in place."""
    B, N, H, d = k_hat.shape
    _dev(k_hat, torch.bfloat16, "k_hat")
    _dev(v_hat, torch.bfloat16, "v_hat", k_hat.shape)
    k = N if idx is None else idx.shape[1]
    _dev(idx, torch.int32, "idx", None if idx is None else (B, k))
    for name, enc, axis in (("k", k_enc, AXIS_TOKEN), ("v", v_enc, AXIS_CHANNEL)):
        _dev(enc[0], torch.uint8, f"{name} codes", (B, k, H, d * bits // 8))
        if bits != 16:
            shp = meta_shape(B, k, H, d, group, axis)
            _dev(enc[1], torch.float16, f"{name} scale", shp)
            _dev(enc[2], torch.float16, f"{name} zero", shp)
    k_rows = v_rows = None
    if mode == DQ_COMPACT:
        k_rows = torch.empty(B, k, H, d, dtype=torch.bfloat16, device=k_hat.device)
        v_rows = torch.empty(B, k, H, d, dtype=torch.bfloat16, device=k_hat.device)
    rc = load().fl_kv_residual_dequant_kv(_p(k_enc[0]), _p(k_enc[1]), _p(k_enc[2]), _p(v_enc[0]), _p(v_enc[1]),
                                          _p(v_enc[2]), _p(idx), k, B, N, H, d, bits, group, mode, _p(k_hat),
                                          _p(v_hat), _p(k_rows), _p(v_rows), _stream())
    _check(rc, "fl_kv_residual_dequant_kv")
    return k_rows, v_rows


def kv_residual_dequant(codes, scale, zero, idx, bits, group, axis, x_hat, mode=DQ_COMPACT):
    """COMPACT: returns the reconstructed rows [B, k, H, d]; COMMIT: updates x_hat in place."""
    B, N, H, d = x_hat.shape
    _dev(x_hat, torch.bfloat16, "x_hat")
    k = N if idx is None else idx.shape[1]
    _dev(idx, torch.int32, "idx", None if idx is None else (B, k))
    _dev(codes, torch.uint8, "codes", (B, k, H, d * bits // 8))
    if bits != 16:
        shp = meta_shape(B, k, H, d, group, axis)
        _dev(scale, torch.float16, "scale", shp)
        _dev(zero, torch.float16, "zero", shp)
    out_rows = None
    if mode == DQ_COMPACT:
        out_rows = torch.empty(B, k, H, d, dtype=torch.bfloat16, device=x_hat.device)
    rc = load().fl_kv_residual_dequant(_p(codes), _p(scale), _p(zero), _p(idx), k, B, N, H, d, bits, group,
                                       axis, mode, _p(x_hat), _p(out_rows), _stream())
    _check(rc, "fl_kv_residual_dequant")
    return out_rows if mode == DQ_COMPACT else x_hat


# ---- (3) attention ----------------------------------------------------------------------------------
def loop_sparse_attn(q_cur, q_prev, k_cache, v_cache, k_new, v_new, slot, rows, cols, window, lse_ref, o,
                     sm_scale=None, ws=None, term_prev=None, mass_prev=None, slot_prev=None, term_out=None,
                     mass_out=None, v16=None):
    """Mass-corrected update of rows `rows` (in place on lse_ref and o).

    term_out/mass_out (fp32 [B, k, H, d] / [B, k, H]) also keep this loop's add terms; term_prev/mass_prev with
    slot_prev (the previous loop's slot map) reuse the previous loop's add terms as the subtract terms, in
    which case q_prev may be None, and k_new/v_new may be None when the caches already hold this loop's rows.
    v16: the fp16 copy of v_cache (given terms over current caches only; fl_loop_sparse_attn_terms_v16)."""
    B, N, H, d = shape = q_cur.shape
    k = rows.shape[1]
    packed = (B, k, H, d)
    reuse = term_prev is not None
    for name, t in (("q_cur", q_cur), ("q_prev", q_prev), ("k_cache", k_cache), ("v_cache", v_cache)):
        _dev(t, torch.bfloat16, name, shape)
    _dev(k_new, torch.bfloat16, "k_new", packed)
    _dev(v_new, torch.bfloat16, "v_new", packed)
    _dev(slot, torch.int32, "slot", (B, N))
    _dev(rows, torch.int32, "rows", (B, k))
    c_list = 0 if cols is None else cols.shape[2]
    _dev(cols, torch.int32, "cols", None if cols is None else (B, H, c_list))
    _dev(lse_ref, torch.float32, "lse_ref", (B, N, H))
    _dev(o, torch.float32, "o", shape)
    k_prev = 0
    if reuse:
        k_prev = term_prev.shape[1]
        _dev(term_prev, torch.float32, "term_prev", (B, k_prev, H, d))
        _dev(mass_prev, torch.float32, "mass_prev", (B, k_prev, H))
        _dev(slot_prev, torch.int32, "slot_prev", (B, N))
    _dev(term_out, torch.float32, "term_out", packed)
    _dev(mass_out, torch.float32, "mass_out", (B, k, H))
    sm_scale = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    lib = load()
    if v16 is not None:
        if not reuse or k_new is not None or v_new is not None:
            raise FlashLoopError("loop_sparse_attn: v16 needs term_prev and current caches (k_new = v_new = None)")
        _dev(v16, torch.float16, "v16", shape)
        rc = lib.fl_loop_sparse_attn_terms_v16(_p(q_cur), _p(k_cache), _p(v_cache), _p(v16), _p(rows), k, _p(cols),
                                               c_list, window, B, N, H, d, sm_scale, _p(lse_ref), _p(o),
                                               _p(term_prev), _p(mass_prev), _p(slot_prev), k_prev, _p(term_out),
                                               _p(mass_out), _stream())
        _check(rc, "fl_loop_sparse_attn_terms_v16")
        return o, lse_ref
    need = lib.fl_loop_sparse_attn_ws(B, N, H, d, k, c_list, window, 0)
    if need and (ws is None or ws.numel() < need):
        ws = torch.empty(need, dtype=torch.uint8, device=q_cur.device)
    if reuse or term_out is not None:
        rc = lib.fl_loop_sparse_attn_terms(_p(q_cur), _p(q_prev), _p(k_cache), _p(v_cache), _p(k_new), _p(v_new),
                                           _p(slot), _p(rows), k, _p(cols), c_list, window, B, N, H, d, sm_scale,
                                           _p(lse_ref), _p(o), _p(term_prev), _p(mass_prev), _p(slot_prev), k_prev,
                                           _p(term_out), _p(mass_out), _p(ws) if need else None, need, _stream())
        _check(rc, "fl_loop_sparse_attn_terms")
    else:
        rc = lib.fl_loop_sparse_attn(_p(q_cur), _p(q_prev), _p(k_cache), _p(v_cache), _p(k_new), _p(v_new),
                                     _p(slot), _p(rows), k, _p(cols), c_list, window, B, N, H, d, sm_scale, 0,
                                     _p(lse_ref), _p(o), _p(ws) if need else None, need, _stream())
        _check(rc, "fl_loop_sparse_attn")
    return o, lse_ref


def attn_kernel_name(pass_, k, c_list, window, B, N, H, d):
    """Name of the kernel an attention pass launches for the shape, or None (fl_attn_kernel_name; host only).
    pass_: PASS_ADD (add pass over current caches), PASS_SUBTRACT or PASS_BOTH."""
    name = load().fl_attn_kernel_name(pass_, k, c_list, window, B, N, H, d)
    return None if name is None else name.decode()


def subtract_terms_supported(k, c_list, window, N, d):
    """Whether fl_loop_subtract_terms covers the shape (a column list of at most 3072 entries)."""
    return bool(load().fl_loop_subtract_terms_supported(k, c_list, window, N, d))


def subtract_terms(q_prev, k_cache, v_cache, rows, cols, window, lse_ref, term_out=None, mass_out=None,
                   sm_scale=None, v16=None):
    """Subtract term and mass of Eq. 7 over the previous loop's state: (term fp32 [B, k, H, d], m fp32 [B, k, H])
    in the row order of `rows` (fl_loop_subtract_terms; with v16, the fp16 copy of v_cache,
    fl_loop_subtract_terms_v16)."""
    B, N, H, d = shape = q_prev.shape
    k = rows.shape[1]
    for name, t in (("q_prev", q_prev), ("k_cache", k_cache), ("v_cache", v_cache)):
        _dev(t, torch.bfloat16, name, shape)
    _dev(rows, torch.int32, "rows", (B, k))
    c_list = 0 if cols is None else cols.shape[2]
    _dev(cols, torch.int32, "cols", None if cols is None else (B, H, c_list))
    _dev(lse_ref, torch.float32, "lse_ref", (B, N, H))
    term_out = torch.empty(B, k, H, d, dtype=torch.float32, device=q_prev.device) if term_out is None else term_out
    mass_out = torch.empty(B, k, H, dtype=torch.float32, device=q_prev.device) if mass_out is None else mass_out
    _dev(term_out, torch.float32, "term_out", (B, k, H, d))
    _dev(mass_out, torch.float32, "mass_out", (B, k, H))
    sm_scale = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    if v16 is not None:
        _dev(v16, torch.float16, "v16", shape)
        rc = load().fl_loop_subtract_terms_v16(_p(q_prev), _p(k_cache), _p(v_cache), _p(v16), _p(rows), k, _p(cols),
                                               c_list, window, B, N, H, d, sm_scale, _p(lse_ref), _p(term_out),
                                               _p(mass_out), _stream())
        _check(rc, "fl_loop_subtract_terms_v16")
        return term_out, mass_out
    rc = load().fl_loop_subtract_terms(_p(q_prev), _p(k_cache), _p(v_cache), _p(rows), k, _p(cols), c_list, window,
                                       B, N, H, d, sm_scale, _p(lse_ref), _p(term_out), _p(mass_out), _stream())
    _check(rc, "fl_loop_subtract_terms")
    return term_out, mass_out


def dense_attn(q, k_cache, v_cache, o=None, lse=None, sm_scale=None):
    """Dense causal loop: returns (o fp32 [B, N, H, d], lse fp32 [B, N, H])."""
    B, N, H, d = q.shape
    for name, t in (("q", q), ("k_cache", k_cache), ("v_cache", v_cache)):
        _dev(t, torch.bfloat16, name, q.shape)
    o = torch.empty(B, N, H, d, dtype=torch.float32, device=q.device) if o is None else o
    lse = torch.empty(B, N, H, dtype=torch.float32, device=q.device) if lse is None else lse
    sm_scale = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    lib = load()
    need = lib.fl_loop_sparse_attn_ws(B, N, H, d, N, 0, 0, ATTN_DENSE)
    ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    rc = lib.fl_loop_sparse_attn(_p(q), None, _p(k_cache), _p(v_cache), None, None, None, None, N, None, 0, 0,
                                 B, N, H, d, sm_scale, ATTN_DENSE, _p(lse), _p(o), _p(ws), need, _stream())
    _check(rc, "fl_loop_sparse_attn(dense)")
    return o, lse


def column_scores(q, k_cache):
    """fp32 column keys [B, H, N] of a dense source loop (64-bit sums inside)."""
    B, N, H, d = q.shape
    _dev(q, torch.bfloat16, "q")
    _dev(k_cache, torch.bfloat16, "k_cache", q.shape)
    lib = load()
    need = lib.fl_column_scores_ws(B, N, H)
    ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    col_key = torch.empty(B, H, N, dtype=torch.float32, device=q.device)
    rc = lib.fl_column_scores(_p(q), _p(k_cache), B, N, H, d, _p(col_key), _p(ws), need, _stream())
    _check(rc, "fl_column_scores")
    return col_key


def select_columns(col_key, n_sink, t):
    """Column list [B, H, min(n_sink, N) + t], ascending."""
    B, H, N = col_key.shape
    _dev(col_key, torch.float32, "col_key")
    ns = min(n_sink, N)
    cols = torch.empty(B, H, ns + t, dtype=torch.int32, device=col_key.device)
    rc = load().fl_select_columns(_p(col_key), B, H, N, n_sink, t, _p(cols), _stream())
    _check(rc, "fl_select_columns")
    return cols


# ---- (6) decode ---------------------------------------------------------------------------------------
def decode_ws(k_cache, cols, c_next):
    """A workspace for decode_step over these shapes (reusable across calls of the same or smaller size)."""
    B, T, H, d = k_cache.shape
    c = 0 if cols is None else cols.shape[2]
    need = load().fl_decode_step_ws(B, T, H, d, c, c_next)
    return torch.empty(max(need, 1), dtype=torch.uint8, device=k_cache.device)


def _decode_args(q, k_cache, v_cache, cols, mass, sub, o, c_next, lse, out):
    B, T, H, d = k_cache.shape
    _dev(q, torch.bfloat16, "q", (B, H, d))
    _dev(k_cache, torch.bfloat16, "k_cache")
    _dev(v_cache, torch.bfloat16, "v_cache", k_cache.shape)
    _dev(o, torch.float32, "o", (B, H, d))
    c = 0 if cols is None else cols.shape[2]
    if cols is not None:
        _dev(cols, torch.int32, "cols", (B, H, c))
        _dev(mass, torch.float32, "mass", (B, H))
        _dev(sub, torch.float32, "sub", (B, H, d))
    _dev(lse, torch.float32, "lse", (B, H))
    cols_next = mass_next = sub_next = None
    if c_next > 0:
        if out is None:
            dev = q.device
            out = (torch.empty(B, H, c_next, dtype=torch.int32, device=dev),
                   torch.empty(B, H, dtype=torch.float32, device=dev),
                   torch.empty(B, H, d, dtype=torch.float32, device=dev))
        cols_next, mass_next, sub_next = out
        _dev(cols_next, torch.int32, "cols_next", (B, H, c_next))
        _dev(mass_next, torch.float32, "mass_next", (B, H))
        _dev(sub_next, torch.float32, "sub_next", (B, H, d))
    return B, T, H, d, c, cols_next, mass_next, sub_next


def decode_step(q, k_cache, v_cache, cols, mass, sub, o, c_next, n_sink=0, window=0, sm_scale=None, lse=None,
                out=None, ws=None):
    """One loop of the decode position T-1.  q bf16 [B, H, d]; caches bf16 [B, T, H, d]; cols int32 [B, H, c]
    (or None for a dense source loop, then mass and sub are unused); o fp32 [B, H, d] updated in place.
    out: optional (cols_next, mass_next, sub_next) to write into; ws: optional workspace (decode_ws).  With
    both given nothing is allocated.  Returns (cols_next [B, H, c_next], mass_next [B, H], sub_next
    [B, H, d]) or Nones when c_next == 0."""
    B, T, H, d, c, cols_next, mass_next, sub_next = _decode_args(q, k_cache, v_cache, cols, mass, sub, o, c_next,
                                                                 lse, out)
    sm_scale = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    lib = load()
    need = lib.fl_decode_step_ws(B, T, H, d, c, c_next)
    if ws is None:
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device=q.device)
    _dev(ws, torch.uint8, "ws")
    rc = lib.fl_decode_step(_p(q), _p(k_cache), _p(v_cache), _p(cols), c, _p(mass), _p(sub), B, T, H, d, sm_scale,
                            _p(o), _p(lse), n_sink, window, c_next, _p(cols_next), _p(mass_next), _p(sub_next),
                            _p(ws), ws.numel(), _stream())
    _check(rc, "fl_decode_step")
    return cols_next, mass_next, sub_next


def decode_step_noalloc(q, k_cache, v_cache, cols, mass, sub, o, c_next, out=None, n_sink=0, window=0,
                        sm_scale=None, lse=None):
    """decode_step without a caller workspace: the library's own device scratch serves as the workspace
    (calls overlapping on one GPU race on it).  Nothing is allocated when `out` is given (or c_next == 0)."""
    B, T, H, d, c, cols_next, mass_next, sub_next = _decode_args(q, k_cache, v_cache, cols, mass, sub, o, c_next,
                                                                 lse, out)
    sm_scale = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    rc = load().fl_decode_step_noalloc(_p(q), _p(k_cache), _p(v_cache), _p(cols), c, _p(mass), _p(sub), B, T, H, d,
                                       sm_scale, _p(o), _p(lse), n_sink, window, c_next, _p(cols_next),
                                       _p(mass_next), _p(sub_next), _stream())
    _check(rc, "fl_decode_step_noalloc")
    return cols_next, mass_next, sub_next


# ---- (7) list pruning for a smaller budget --------------------------------------------------------------
def prune_columns(q, k_cache, rows, cols, lse_ref, n_sink, t_next, sm_scale=None):
    """Keep the sinks and the t_next list entries that loop r's updated rows gave the most probability mass.
    q, k_cache bf16 [B, N, H, d] (loop r); rows int32 [B, k] (or None when k = 0); cols int32 [B, H, c_list];
    lse_ref fp32 [B, N, H].  Returns (cols_next int32 [B, H, ns + t_next], col_key fp32 [B, H, c_list - ns])."""
    B, N, H, d = k_cache.shape
    _dev(q, torch.bfloat16, "q", k_cache.shape)
    _dev(k_cache, torch.bfloat16, "k_cache")
    c_list = cols.shape[2]
    _dev(cols, torch.int32, "cols", (B, H, c_list))
    _dev(lse_ref, torch.float32, "lse_ref", (B, N, H))
    k = 0 if rows is None else rows.shape[1]
    if rows is not None:
        _dev(rows, torch.int32, "rows", (B, k))
    ns = min(n_sink, c_list)
    dev = q.device
    col_key = torch.empty(B, H, c_list - ns, dtype=torch.float32, device=dev)
    cols_next = torch.empty(B, H, ns + t_next, dtype=torch.int32, device=dev)
    sm_scale = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    lib = load()
    need = lib.fl_prune_columns_ws(B, H, k, c_list, n_sink)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    rc = lib.fl_prune_columns(_p(q), _p(k_cache), _p(rows), k, _p(cols), c_list, _p(lse_ref), B, N, H, d,
                              sm_scale, n_sink, t_next, _p(col_key) if c_list > ns else None, _p(cols_next),
                              _p(ws), need, _stream())
    _check(rc, "fl_prune_columns")
    return cols_next, col_key


# ---- (8) recent tokens kept in bf16 --------------------------------------------------------------------
def kv_keep_recent(x_cur, idx, tail, cache=None, rows=None):
    """Store the active rows i >= N - tail exactly: cache [B, N, H, d] at i and/or the compact rows
    [B, k, H, d] at their position (x_cur bf16 [B, N, H, d]; idx int32 [B, k] or None for every row)."""
    B, N, H, d = x_cur.shape
    _dev(x_cur, torch.bfloat16, "x_cur")
    k = N if idx is None else idx.shape[1]
    _dev(idx, torch.int32, "idx", None if idx is None else (B, k))
    _dev(cache, torch.bfloat16, "cache", None if cache is None else x_cur.shape)
    _dev(rows, torch.bfloat16, "rows", None if rows is None else (B, k, H, d))
    rc = load().fl_kv_keep_recent(_p(x_cur), _p(idx), k, B, N, H, d, tail, _p(cache), _p(rows), _stream())
    _check(rc, "fl_kv_keep_recent")


# ---- (9) rotary positions -------------------------------------------------------------------------------
_DTYPES = {torch.bfloat16: 0, torch.float16: 1}
_FORMATS = {torch.int8: 0, torch.float8_e4m3fn: 1}
_FORMATS4 = {torch.float16: 0, torch.uint8: 1}       # by the type of the groups' numbers


# (As above, a tensor that passes its checks passes them in one expression: a call's host time is that of its launch.)
if hasattr(torch._C, "_cuda_getDevice"):
    _current = torch._C._cuda_getDevice
else:
    _current = torch.cuda.current_device


def _here(t, name):
    """The device number of t: the calls below launch on the current device's stream, so their tensors have to be there."""
    if not t.is_cuda:
        raise FlashLoopError(f"{name} must be a device tensor")
    at = t.get_device()
    if at != _current():
        raise FlashLoopError(f"{name} is on cuda:{at}, but the current device is cuda:{_current()}")
    return at


def _on(t, at, dtype, name, shape=None):
    if t is None or (t.dtype is dtype and t.get_device() == at and t.is_contiguous() and (shape is None or t.shape == shape)):
        return
    _dev(t, dtype, name, shape)
    raise FlashLoopError(f"{name} is on {t.device}, the call's other tensors on cuda:{at}")


def _rows(t, at, dtype, name, shape=None):
    """Elements between the rows of [T, H, d], whose heads are dense."""
    if (shape is None and t.dim() != 3) or (shape is not None and t.shape != shape):
        raise FlashLoopError(f"{name} must have shape {'[T, H, d]' if shape is None else tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype is not dtype or dtype not in _DTYPES:
        raise FlashLoopError(f"{name} must be {dtype if dtype in _DTYPES else 'bfloat16 or float16'}, got {t.dtype}")
    if t.get_device() != at:
        raise FlashLoopError(f"{name} is on {t.device}, the call's other tensors on cuda:{at}")
    (T, H, d), (row, head, one) = t.shape, t.stride()
    if (one != 1 and d > 1) or (head != d and H > 1):
        raise FlashLoopError(f"the heads of a row of {name} must be dense, got strides {t.stride()}")
    return row if T > 1 else H * d


def _choice(value, of, name):
    number = of.get(value)
    if number is None:
        raise FlashLoopError(f"{name} must be one of {', '.join(of)}, got {value!r}")
    return number


def _counts(**counts):
    """Refuses what a C int does not hold (it would be passed modulo 2^32).  Callers test that first, in one expression."""
    for name, n in counts.items():
        if n >> 31:
            raise FlashLoopError(f"{name} must be in [0, 2^31), got {n}")


def _turns(table, at):
    """(n_pos, rot) of a rotary table, (0, 0) without one."""
    if table is None:
        return 0, 0
    _on(table, at, torch.float32, "table")
    if table.dim() != 3 or table.shape[2] != 2:
        raise FlashLoopError(f"table must have shape [n_pos, rot / 2, 2], got {tuple(table.shape)}")
    n_pos, half, _ = table.shape
    return n_pos, 2 * half


def rope_table(n_pos, rot, base=10000.0, scaling="none", factor=1.0, orig_len=0, low=1.0, high=32.0, out=None, device=None):
    """Cosines and sines of positions 0 .. n_pos-1: fp32 [n_pos, rot / 2, 2].  scaling: "none", "linear" (positions divided
    by factor), "ntk" (a larger base, so that the lowest frequency is divided by factor) or "yarn" (frequencies that turn
    fewer than low times within orig_len positions divided by factor, those above high kept, and the table multiplied by
    1 + 0.1 ln(factor)).  On `device` (out's, or the current one)."""
    how = _choice(scaling, ROPE_SCALING, "scaling")
    _counts(n_pos=n_pos, rot=rot)
    if out is None:
        out = torch.empty(n_pos, rot // 2, 2, dtype=torch.float32, device="cuda" if device is None else device)
        _here(out, "device")
    else:
        _on(out, _here(out, "out"), torch.float32, "out", (n_pos, rot // 2, 2))
    rc = load().fl_rope_table(n_pos, rot, base, how, factor, orig_len, low, high, _p(out), _stream())
    _check(rc, "fl_rope_table")
    return out


def rope(x, table, pos=None, layout="half", inverse=False, out=None):
    """The rows of x (bf16 or fp16 [T, H, d], any row stride that is a multiple of 8) with their heads' first rot channels
    turned by the positions pos (int32 [T]; None: 0 .. T-1).  inverse=True turns back: the gradient of x from that of the
    result.  out: where to write (x itself: in place).  A dense [B, N, H, d] state is x.view(B * N, H, d)."""
    at, dtype = _here(x, "x"), x.dtype
    xs = _rows(x, at, dtype, "x")
    n_pos, rot = _turns(table, at)
    if table is None:
        raise FlashLoopError("rope needs a table")
    T, H, d = x.shape
    if (T | n_pos) >> 31:
        _counts(T=T, n_pos=n_pos)
    _on(pos, at, torch.int32, "pos", (T,))
    if out is None:
        out, ys = x.new_empty((T, H, d)), H * d
    else:
        ys = _rows(out, at, dtype, "out", x.shape)
    rc = (_lib or load()).fl_rope(x.data_ptr(), xs, _p(pos), table.data_ptr(), n_pos, rot, _choice(layout, ROPE_LAYOUT, "layout"),
                                  1 if inverse else 0, _DTYPES[dtype], T, H, d, out.data_ptr(), ys, _stream())
    if rc:
        _check(rc, "fl_rope")
    return out


# ---- (10) the paged 8-bit cache ---------------------------------------------------------------------------
def _paged(at, T, cu, lens, block_table, k_cache, v_cache, k_scale, v_scale, Hkv, d):
    """(B, max_pages, num_pages, page, format) of a ragged batch over a cache."""
    if block_table.dim() != 2 or k_cache.dim() != 4:
        raise FlashLoopError("block_table must be [B, max_pages] and the caches [num_pages, Hkv, page, d]")
    code = k_cache.dtype
    if code not in _FORMATS:
        raise FlashLoopError(f"the caches must be int8 or float8_e4m3fn, got {code}")
    B, max_pages = block_table.shape
    if B == 0:
        raise FlashLoopError("a batch has at least one sequence")
    shape = num_pages, _, page, _ = k_cache.shape
    if (T | B | max_pages | num_pages) >> 31:
        _counts(T=T, B=B, max_pages=max_pages, num_pages=num_pages)
    if (shape[1] != Hkv or shape[3] != d or v_cache.dtype is not code or v_cache.shape != shape
            or not (k_cache.is_contiguous() and v_cache.is_contiguous() and k_cache.get_device() == v_cache.get_device() == at)):
        for name, c in (("k_cache", k_cache), ("v_cache", v_cache)):
            _on(c, at, code, name, (num_pages, Hkv, page, d))
    if not (k_scale.dtype is v_scale.dtype is torch.float32 and cu.dtype is lens.dtype is block_table.dtype is torch.int32
            and k_scale.get_device() == v_scale.get_device() == cu.get_device() == lens.get_device() == block_table.get_device() == at
            and k_scale.shape == v_scale.shape == (num_pages, Hkv) and cu.shape == (B + 1,) and lens.shape == (B,)
            and k_scale.is_contiguous() and v_scale.is_contiguous() and cu.is_contiguous() and lens.is_contiguous()
            and block_table.is_contiguous()):
        _on(k_scale, at, torch.float32, "k_scale", (num_pages, Hkv))
        _on(v_scale, at, torch.float32, "v_scale", (num_pages, Hkv))
        _on(cu, at, torch.int32, "cu", (B + 1,))
        _on(lens, at, torch.int32, "lens", (B,))
        _on(block_table, at, torch.int32, "block_table")
    return B, max_pages, num_pages, page, _FORMATS[code]


def paged_cache(num_pages, Hkv, page, d, dtype=torch.int8, device="cuda"):
    """An empty cache: (k_cache, v_cache [num_pages, Hkv, page, d] of int8 or float8_e4m3fn codes, k_scale, v_scale fp32
    [num_pages, Hkv]).  Pages need no clearing, here or when they are given to another sequence."""
    if dtype not in _FORMATS:
        raise FlashLoopError(f"the caches must be int8 or float8_e4m3fn, got {dtype}")
    codes = [torch.empty(num_pages, Hkv, page, d, dtype=dtype, device=device) for _ in range(2)]
    return (*codes, *(torch.zeros(num_pages, Hkv, dtype=torch.float32, device=device) for _ in range(2)))


def paged_append(k, v, cu, lens, block_table, k_cache, v_cache, k_scale, v_scale, table=None, layout="half"):
    """Store the new positions of a ragged batch.  k, v: bf16 or fp16 [T, Hkv, d], any row stride that is a multiple of 8;
    rows cu[b] .. cu[b+1]-1 (int32 [B + 1]) are the last positions of sequence b, whose length with them is lens[b] (int32
    [B]); block_table: int32 [B, max_pages], its pages.  With a rotary table the keys are turned by their positions on the
    way.  The caches (paged_cache) are updated in place; the scale of a page and head covers what the page holds of the
    sequence, and doubles (its earlier codes halve) when a new position needs it."""
    at, dtype = _here(k, "k"), k.dtype
    ks = _rows(k, at, dtype, "k")
    T, Hkv, d = k.shape
    vs = _rows(v, at, dtype, "v", k.shape)
    B, max_pages, num_pages, page, fmt = _paged(at, T, cu, lens, block_table, k_cache, v_cache, k_scale, v_scale, Hkv, d)
    n_pos, rot = _turns(table, at)
    if n_pos >> 31:
        _counts(n_pos=n_pos)
    rc = (_lib or load()).fl_paged_append(
        k.data_ptr(), ks, v.data_ptr(), vs, _DTYPES[dtype], cu.data_ptr(), lens.data_ptr(), B, T, Hkv, d, _p(table), n_pos, rot,
        _choice(layout, ROPE_LAYOUT, "layout"), block_table.data_ptr(), max_pages, num_pages, page, fmt, k_cache.data_ptr(),
        v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), _stream())
    if rc:
        _check(rc, "fl_paged_append")


# ---- (11) attention over the paged cache ------------------------------------------------------------------
def paged_attn(q, cu, lens, block_table, k_cache, v_cache, k_scale, v_scale, table=None, layout="half", sm_scale=None,
               window=0, n_sink=0, max_q=None, max_len=0, out=None, lse=None, ws=None):
    """Causal attention of the last positions of every sequence over its cached ones (after paged_append of the same
    batch): q bf16 or fp16 [T, Hq, d], any row stride that is a multiple of 8, turned by its positions when a rotary table is
    given; Hq a multiple of the cache's heads.  window > 0: a row at position i sees j > i - window and j < n_sink alone.
    max_q, max_len: the largest number of new positions and the largest length of a sequence, as far as known (they choose
    the kernel, not the result; default: an even batch, as long as the block table allows).  lse: optional fp32 [T, Hq] to
    write the log-normalisers to.  ws: optional uint8 workspace (paged_attn_ws).  Returns out [T, Hq, d]; rows behind cu[B] of
    a given out are left as they were."""
    at, dtype = _here(q, "q"), q.dtype
    qs = _rows(q, at, dtype, "q")
    T, Hq, d = q.shape
    Hkv = k_cache.shape[1] if k_cache.dim() == 4 else 0
    B, max_pages, num_pages, page, fmt = _paged(at, T, cu, lens, block_table, k_cache, v_cache, k_scale, v_scale, Hkv, d)
    n_pos, rot = _turns(table, at)
    if out is None:
        out, os_ = q.new_empty((T, Hq, d)), Hq * d
    else:
        os_ = _rows(out, at, dtype, "out", q.shape)
    _on(lse, at, torch.float32, "lse", (T, Hq))
    max_q = -(-T // B) if max_q is None else max_q
    if (window | n_sink | max_q | max_len | n_pos) >> 31:
        _counts(window=window, n_sink=n_sink, max_q=max_q, max_len=max_len, n_pos=n_pos)
    lib = _lib or load()
    if ws is None:
        need = lib.fl_paged_attn_ws(B, T, Hq, Hkv, d, page, max_pages, window, n_sink, max_q, max_len)
        ws = lens.new_empty(need, dtype=torch.uint8) if need else None
    else:
        _on(ws, at, torch.uint8, "ws")
    rc = lib.fl_paged_attn(
        q.data_ptr(), qs, _DTYPES[dtype], cu.data_ptr(), lens.data_ptr(), B, T, Hq, Hkv, d, _p(table), n_pos, rot,
        _choice(layout, ROPE_LAYOUT, "layout"), block_table.data_ptr(), max_pages, num_pages, page, fmt, k_cache.data_ptr(),
        v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), 1.0 / math.sqrt(d) if sm_scale is None else sm_scale, window,
        n_sink, max_q, max_len, out.data_ptr(), os_, _p(lse), _p(ws), 0 if ws is None else ws.numel(), _stream())
    if rc:
        _check(rc, "fl_paged_attn")
    return out


def paged_attn_ws(q, block_table, k_cache, window=0, n_sink=0, max_q=None, max_len=0):
    """A workspace for paged_attn over these shapes and hints (None when it needs none)."""
    T, Hq, d = q.shape
    B, max_pages = max(1, block_table.shape[0]), block_table.shape[1]
    max_q = -(-T // B) if max_q is None else max_q
    _counts(T=T, B=B, max_pages=max_pages, window=window, n_sink=n_sink, max_q=max_q, max_len=max_len)
    need = load().fl_paged_attn_ws(B, T, Hq, k_cache.shape[1], d, k_cache.shape[2], max_pages, window, n_sink, max_q, max_len)
    return torch.empty(need, dtype=torch.uint8, device=q.device) if need else None


# ---- (12) attention of packed prompts ---------------------------------------------------------------------
def packed_attn(q, k, v, cu_q, cu_k=None, table=None, layout="half", sm_scale=None, window=0, n_sink=0, max_k=0, out=None, lse=None,
                ws=None):
    """Causal attention of packed sequences: q bf16 or fp16 [Tq, Hq, d], k and v [Tk, Hkv, d] of its type, any row strides that
    are multiples of 8; Hq a multiple of Hkv.  Sequence b has the query rows cu_q[b] .. cu_q[b+1]-1 (int32 [B + 1]) and the key rows
    cu_k[b] .. cu_k[b+1]-1 (default: cu_q, whole prompts); its queries are the last of its positions.  window > 0: a row at position
    i sees j > i - window and j < n_sink alone.  With a rotary table the queries (not the keys) are turned by their positions, as
    rope leaves them.  max_k: the largest number of keys of a sequence, as far as known (it chooses how the work is cut, not the
    result; default: an even batch).  lse: optional fp32 [Tq, Hq] to write the log-normalisers to.  ws: optional uint8 workspace
    (packed_attn_ws).  Returns out [Tq, Hq, d]; rows behind cu_q[B] of a given out are left as they were."""
    at, dtype = _here(q, "q"), q.dtype
    qs = _rows(q, at, dtype, "q")
    Tq, Hq, d = q.shape
    ks = _rows(k, at, dtype, "k")
    Tk, Hkv, dk = shape = k.shape
    vs = _rows(v, at, dtype, "v", shape)
    if dk != d:
        raise FlashLoopError(f"k must have heads of {d} channels as q has, got {dk}")
    if cu_k is None:
        cu_k = cu_q
    if cu_q.dim() != 1 or cu_q.shape[0] < 2:
        raise FlashLoopError(f"cu_q must have shape [B + 1] for at least one sequence, got {tuple(cu_q.shape)}")
    B = cu_q.shape[0] - 1
    _on(cu_q, at, torch.int32, "cu_q")
    _on(cu_k, at, torch.int32, "cu_k", (B + 1,))
    n_pos, rot = _turns(table, at)
    if out is None:
        out, os_ = q.new_empty((Tq, Hq, d)), Hq * d
    else:
        os_ = _rows(out, at, dtype, "out", q.shape)
    _on(lse, at, torch.float32, "lse", (Tq, Hq))
    if (window | n_sink | max_k | n_pos | Tq | Tk | B) >> 31:
        _counts(window=window, n_sink=n_sink, max_k=max_k, n_pos=n_pos, Tq=Tq, Tk=Tk, B=B)
    lib = _lib or load()
    if ws is None:
        need = lib.fl_packed_attn_ws(B, Tq, Tk, Hq, Hkv, d, window, n_sink, max_k)
        ws = cu_q.new_empty(need, dtype=torch.uint8) if need else None
    else:
        _on(ws, at, torch.uint8, "ws")
    rc = lib.fl_packed_attn(q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs, _DTYPES[dtype], cu_q.data_ptr(), cu_k.data_ptr(), B,
                            Tq, Tk, Hq, Hkv, d, _p(table), n_pos, rot, _choice(layout, ROPE_LAYOUT, "layout"),
                            1.0 / math.sqrt(d) if sm_scale is None else sm_scale, window, n_sink, max_k, out.data_ptr(), os_, _p(lse),
                            _p(ws), 0 if ws is None else ws.numel(), _stream())
    if rc:
        _check(rc, "fl_packed_attn")
    return out


def packed_attn_ws(q, k, B, window=0, n_sink=0, max_k=0):
    """A workspace for packed_attn over these shapes and hints (None when it needs none)."""
    (Tq, Hq, d), (Tk, Hkv, _) = q.shape, k.shape
    _counts(Tq=Tq, Tk=Tk, B=B, window=window, n_sink=n_sink, max_k=max_k)
    need = load().fl_packed_attn_ws(B, Tq, Tk, Hq, Hkv, d, window, n_sink, max_k)
    return torch.empty(need, dtype=torch.uint8, device=q.device) if need else None


# ---- (13) the paged 4-bit cache ---------------------------------------------------------------------------
KV4_FORMAT = {"int4": torch.float16, "e2m1": torch.uint8}


def paged4_cache(num_pages, Hkv, page, d, fmt="int4", device="cuda"):
    """An empty 4-bit cache: (k_cache, v_cache uint8 [num_pages, Hkv, page, d / 2], k_meta, v_meta).  Groups of 32 channels of a
    position and head have numbers of their own: "int4" fp16 [num_pages, Hkv, page, d / 32, 2] (scale, zero), "e2m1" uint8
    [num_pages, Hkv, page, d / 32] exponents + 127.  Pages need no clearing, here or when they are given to another sequence."""
    kind = _choice(fmt, KV4_FORMAT, "fmt")
    shape = (num_pages, Hkv, page, d // 32) + ((2,) if fmt == "int4" else ())
    return (*(torch.empty(num_pages, Hkv, page, d // 2, dtype=torch.uint8, device=device) for _ in range(2)),
            *(torch.empty(shape, dtype=kind, device=device) for _ in range(2)))


def _paged4(at, T, cu, lens, block_table, k_cache, v_cache, k_meta, v_meta, Hkv, d):
    """(B, max_pages, num_pages, page, format) of a ragged batch over a 4-bit cache."""
    if block_table.dim() != 2 or k_cache.dim() != 4:
        raise FlashLoopError("block_table must be [B, max_pages] and the caches [num_pages, Hkv, page, d / 2]")
    kind = k_meta.dtype
    if kind not in _FORMATS4:
        raise FlashLoopError(f"k_meta must be float16 (int4) or uint8 (e2m1), got {kind}")
    B, max_pages = block_table.shape
    if B == 0:
        raise FlashLoopError("a batch has at least one sequence")
    shape = num_pages, _, page, _ = k_cache.shape
    if (T | B | max_pages | num_pages) >> 31:
        _counts(T=T, B=B, max_pages=max_pages, num_pages=num_pages)
    groups = (num_pages, Hkv, page, d // 32, 2) if kind is torch.float16 else (num_pages, Hkv, page, d // 32)
    if not (shape[1] == Hkv and shape[3] * 2 == d and k_cache.dtype is v_cache.dtype is torch.uint8 and v_cache.shape == shape
            and v_meta.dtype is kind and k_meta.shape == v_meta.shape == groups
            and cu.dtype is lens.dtype is block_table.dtype is torch.int32 and cu.shape == (B + 1,) and lens.shape == (B,)
            and k_cache.get_device() == v_cache.get_device() == k_meta.get_device() == v_meta.get_device() == cu.get_device()
            == lens.get_device() == block_table.get_device() == at
            and k_cache.is_contiguous() and v_cache.is_contiguous() and k_meta.is_contiguous() and v_meta.is_contiguous()
            and cu.is_contiguous() and lens.is_contiguous() and block_table.is_contiguous()):
        for name, c in (("k_cache", k_cache), ("v_cache", v_cache)):
            _on(c, at, torch.uint8, name, (num_pages, Hkv, page, d // 2))
        for name, c in (("k_meta", k_meta), ("v_meta", v_meta)):
            _on(c, at, kind, name, groups)
        _on(cu, at, torch.int32, "cu", (B + 1,))
        _on(lens, at, torch.int32, "lens", (B,))
        _on(block_table, at, torch.int32, "block_table")
        raise FlashLoopError(f"the caches hold heads of {2 * shape[3]} channels, not {d}")
    return B, max_pages, num_pages, page, _FORMATS4[kind]


def paged4_append(k, v, cu, lens, block_table, k_cache, v_cache, k_meta, v_meta, table=None, layout="half", k_rows=None, v_rows=None):
    """Store the new positions of a ragged batch in 4 bits; the batch, the block table and the rotary table are those of
    paged_append, the cache is paged4_cache's and updated in place.  k_rows, v_rows: optional [T, Hkv, d] of k's type to write the
    rows to that the codes stand for (k and v themselves: in place), as paged4_read gives them: the attention of a whole prompt over
    them (packed_attn) sees what later steps read."""
    at, dtype = _here(k, "k"), k.dtype
    ks = _rows(k, at, dtype, "k")
    T, Hkv, d = shape = k.shape
    vs = _rows(v, at, dtype, "v", shape)
    B, max_pages, num_pages, page, fmt = _paged4(at, T, cu, lens, block_table, k_cache, v_cache, k_meta, v_meta, Hkv, d)
    n_pos, rot = _turns(table, at)
    if n_pos >> 31:
        _counts(n_pos=n_pos)
    krs = 0 if k_rows is None else _rows(k_rows, at, dtype, "k_rows", shape)
    vrs = 0 if v_rows is None else _rows(v_rows, at, dtype, "v_rows", shape)
    rc = (_lib or load()).fl_paged4_append(
        k.data_ptr(), ks, v.data_ptr(), vs, _DTYPES[dtype], cu.data_ptr(), lens.data_ptr(), B, T, Hkv, d, _p(table), n_pos, rot,
        _choice(layout, ROPE_LAYOUT, "layout"), block_table.data_ptr(), max_pages, num_pages, page, fmt, k_cache.data_ptr(),
        v_cache.data_ptr(), k_meta.data_ptr(), v_meta.data_ptr(), _p(k_rows), krs, _p(v_rows), vrs, _stream())
    if rc:
        _check(rc, "fl_paged4_append")


# ---- (14) reading the 4-bit cache back ----------------------------------------------------------------------
def paged4_read(cu, lens, block_table, k_cache, v_cache, k_meta, v_meta, T, dtype=torch.bfloat16, k_out=None, v_out=None):
    """Positions of a ragged batch out of a 4-bit cache: rows cu[b] .. cu[b+1]-1 of T are the last positions of sequence b, whose
    length is lens[b] (cu the cumulative lengths: all of it).  Returns (k, v) [T, Hkv, d] of `dtype` (k_out's or v_out's where one
    is given; rows of no sequence are left as they were).  A dense [B, N, H, d] state: k_out=state.view(B * N, H, d)."""
    at = _here(k_cache, "k_cache")
    if k_cache.dim() != 4:
        raise FlashLoopError("the caches must be [num_pages, Hkv, page, d / 2]")
    Hkv, d = k_cache.shape[1], 2 * k_cache.shape[3]
    if T >> 31:
        _counts(T=T)
    for name, given in (("k_out", k_out), ("v_out", v_out)):
        dtype = dtype if given is None else given.dtype
    if dtype not in _DTYPES:
        raise FlashLoopError(f"dtype must be bfloat16 or float16, got {dtype}")
    B, max_pages, num_pages, page, fmt = _paged4(at, T, cu, lens, block_table, k_cache, v_cache, k_meta, v_meta, Hkv, d)
    k_out = k_cache.new_empty((T, Hkv, d), dtype=dtype) if k_out is None else k_out
    v_out = k_cache.new_empty((T, Hkv, d), dtype=dtype) if v_out is None else v_out
    ks, vs = _rows(k_out, at, dtype, "k_out", (T, Hkv, d)), _rows(v_out, at, dtype, "v_out", (T, Hkv, d))
    rc = (_lib or load()).fl_paged4_read(
        cu.data_ptr(), lens.data_ptr(), B, T, Hkv, d, block_table.data_ptr(), max_pages, num_pages, page, fmt, k_cache.data_ptr(),
        v_cache.data_ptr(), k_meta.data_ptr(), v_meta.data_ptr(), _DTYPES[dtype], k_out.data_ptr(), ks, v_out.data_ptr(), vs, _stream())
    if rc:
        _check(rc, "fl_paged4_read")
    return k_out, v_out


# ---- (15) attention over the 4-bit cache --------------------------------------------------------------------
def paged4_attn(q, cu, lens, block_table, k_cache, v_cache, k_meta, v_meta, table=None, layout="half", sm_scale=None,
                window=0, n_sink=0, max_q=None, max_len=0, out=None, lse=None, ws=None):
    """paged_attn over a 4-bit cache (after paged4_append of the same batch): its arguments, hints and result."""
    at, dtype = _here(q, "q"), q.dtype
    qs = _rows(q, at, dtype, "q")
    T, Hq, d = q.shape
    Hkv = k_cache.shape[1] if k_cache.dim() == 4 else 0
    B, max_pages, num_pages, page, fmt = _paged4(at, T, cu, lens, block_table, k_cache, v_cache, k_meta, v_meta, Hkv, d)
    n_pos, rot = _turns(table, at)
    if out is None:
        out, os_ = q.new_empty((T, Hq, d)), Hq * d
    else:
        os_ = _rows(out, at, dtype, "out", q.shape)
    _on(lse, at, torch.float32, "lse", (T, Hq))
    max_q = -(-T // B) if max_q is None else max_q
    if (window | n_sink | max_q | max_len | n_pos) >> 31:
        _counts(window=window, n_sink=n_sink, max_q=max_q, max_len=max_len, n_pos=n_pos)
    lib = _lib or load()
    if ws is None:
        need = lib.fl_paged4_attn_ws(B, T, Hq, Hkv, d, page, max_pages, window, n_sink, max_q, max_len)
        ws = lens.new_empty(need, dtype=torch.uint8) if need else None
    else:
        _on(ws, at, torch.uint8, "ws")
    rc = lib.fl_paged4_attn(
        q.data_ptr(), qs, _DTYPES[dtype], cu.data_ptr(), lens.data_ptr(), B, T, Hq, Hkv, d, _p(table), n_pos, rot,
        _choice(layout, ROPE_LAYOUT, "layout"), block_table.data_ptr(), max_pages, num_pages, page, fmt, k_cache.data_ptr(),
        v_cache.data_ptr(), k_meta.data_ptr(), v_meta.data_ptr(), 1.0 / math.sqrt(d) if sm_scale is None else sm_scale, window,
        n_sink, max_q, max_len, out.data_ptr(), os_, _p(lse), _p(ws), 0 if ws is None else ws.numel(), _stream())
    if rc:
        _check(rc, "fl_paged4_attn")
    return out


def paged4_attn_ws(q, block_table, k_cache, window=0, n_sink=0, max_q=None, max_len=0):
    """A workspace for paged4_attn over these shapes and hints (None when it needs none)."""
    T, Hq, d = q.shape
    B, max_pages = max(1, block_table.shape[0]), block_table.shape[1]
    max_q = -(-T // B) if max_q is None else max_q
    _counts(T=T, B=B, max_pages=max_pages, window=window, n_sink=n_sink, max_q=max_q, max_len=max_len)
    need = load().fl_paged4_attn_ws(B, T, Hq, k_cache.shape[1], d, k_cache.shape[2], max_pages, window, n_sink, max_q, max_len)
    return torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
