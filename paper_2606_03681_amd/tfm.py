"""Thin ctypes binding of libtfmlayer.so (C ABI in include/tfm_layer.h, include/tfm_ends.h,
include/tfm_vocab.h, include/tfm_cache.h and include/tfm_optim.h).

Argument marshalling only: every step of the layer runs in the library's HIP kernels.  torch
supplies device memory and the stream.  There is no fallback: if the library is missing, every
call raises.
"""

import ctypes
import os
import struct

import numpy as np

# TFM_LIB may name another build of the same library (the host-sanitizer build of build.py)
_LIB_PATH = os.environ.get("TFM_LIB") or \
    os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtfmlayer.so")
_lib = None

TFM_F32, TFM_BF16 = 0, 1
TFM_BLOCK_POSTNORM, TFM_BLOCK_PRENORM = 0, 1
ERRORS = {
    -1: "TFM_ERR_DIMS", -2: "TFM_ERR_HEAD_DIM", -3: "TFM_ERR_NTRAIN", -4: "TFM_ERR_MASK",
    -5: "TFM_ERR_POINTER", -6: "TFM_ERR_HIP", -7: "TFM_ERR_BUFFER",
}
EXPORTS = ("tfm_layer_param_count", "tfm_layer_saved_bytes", "tfm_layer_workspace_bytes",
           "tfm_layer_fwd", "tfm_layer_fwd_noalloc", "tfm_layer_bwd", "tfm_thinking_rows_fwd",
           "tfm_thinking_rows_bwd",
           "tfm_infer_workspace_bytes", "tfm_infer_cache_bytes", "tfm_layer_fwd_context",
           "tfm_layer_fwd_query", "tfm_last_error", "tfm_prof_enable", "tfm_prof_collect",
           "tfm_prof_step", "tfm_prof_item_bwd_fused_rows", "tfm_prof_item_bwd_columns",
           "tfm_ends_param_count", "tfm_ends_workspace_bytes", "tfm_encode_fwd",
           "tfm_encode_bwd", "tfm_decode_fwd", "tfm_decode_loss", "tfm_decode_bwd",
           "tfm_embed_workspace_bytes", "tfm_embed_fwd", "tfm_embed_bwd",
           "tfm_distill_workspace_bytes", "tfm_distill_loss", "tfm_sample",
           "tfm_adjust_logits", "tfm_cache8_bytes", "tfm_cache8_append",
           "tfm_cache8_attend_workspace_bytes", "tfm_cache8_attend", "tfm_infer_cache8_bytes",
           "tfm_infer8_workspace_bytes", "tfm_layer_fwd_context8", "tfm_layer_fwd_query8",
           "tfm_clip_workspace_bytes",
           "tfm_clip_scale", "tfm_sfadamw_step", "tfm_muon_workspace_bytes", "tfm_muon_step")


class TfmError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{ERRORS.get(code, code)}: {msg}")
        self.code = code


class tfm_dims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "R", "C", "E", "heads", "H", "dtype",
                                               "block")] + [("decay", ctypes.c_float)]


def make_dims(B, R, C, E, heads, H, dtype, block="post", decay=1.0):
    dt = {"f32": TFM_F32, "bf16": TFM_BF16}.get(dtype, dtype)
    bk = {"post": TFM_BLOCK_POSTNORM, "pre": TFM_BLOCK_PRENORM}.get(block, block)
    return tfm_dims(int(B), int(R), int(C), int(E), int(heads), int(H), int(dt), int(bk),
                    float(decay))


class tfm_ends(ctypes.Structure):
    _fields_ = [("G", ctypes.c_int32), ("offsets", ctypes.c_int32 * 8)] + \
        [(n, ctypes.c_int32) for n in ("F", "T", "Hd", "K", "decode_mean")]


def make_ends(G, offsets, F, T, Hd, K, decode_mean):
    offs = list(offsets)
    if len(offs) != G or G > 8:
        raise ValueError(f"need G = {G} <= 8 offsets, got {offs}")
    arr = (ctypes.c_int32 * 8)(*(offs + [0] * (8 - len(offs))))
    return tfm_ends(int(G), arr, int(F), int(T), int(Hd), int(K), int(bool(decode_mean)))


class tfm_sfadamw(ctypes.Structure):
    _fields_ = [(n, ctypes.c_float) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")] + \
        [("warmup", ctypes.c_int32)]


class tfm_muon(ctypes.Structure):
    _fields_ = [(n, ctypes.c_float) for n in ("lr", "momentum", "weight_decay")] + \
        [("nesterov", ctypes.c_int32), ("ns_steps", ctypes.c_int32)]


_DTYPES = {"f32": TFM_F32, "bf16": TFM_BF16}


class tfm_embed(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32 * 3)] + \
        [(n, ctypes.c_int32) for n in ("E", "V", "dtype", "table_dtype")] + \
        [("scale", ctypes.c_float), ("stride", ctypes.c_int64 * 3)]


def make_embed(n, stride, E, V, dtype, table_dtype="f32", scale=1.0):
    """n: shape (n0, n1, n2) of the ids; stride: elements between rows along each of its axes."""
    if len(n) != 3 or len(stride) != 3:
        raise ValueError(f"need three sizes and three strides, got {n} and {stride}")
    return tfm_embed(tuple(map(int, n)), int(E), int(V), int(_DTYPES.get(dtype, dtype)),
                     int(_DTYPES.get(table_dtype, table_dtype)), float(scale),
                     tuple(map(int, stride)))


class tfm_distill(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("N", "V", "k", "dtype", "tail")] + \
        [("temperature", ctypes.c_float), ("alpha", ctypes.c_float), ("ld", ctypes.c_int64)]


def make_distill(N, V, k, ld, dtype, temperature=1.0, alpha=1.0, tail=False):
    return tfm_distill(int(N), int(V), int(k), int(_DTYPES.get(dtype, dtype)), int(tail),
                       float(temperature), float(alpha), int(ld))


class tfm_sampling(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("N", "V", "dtype")] + [("ld", ctypes.c_int64)]


def make_sampling(N, V, ld, dtype):
    return tfm_sampling(int(N), int(V), int(_DTYPES.get(dtype, dtype)), int(ld))


# packed, these structures take half the time that filling their fields does (1.2 and 2.8 us)
_ADJUST = struct.Struct("5i5q")
_ROWS = struct.Struct("4i3q3q")
_QUERY = struct.Struct("7if3q3q")


class tfm_adjust(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("N", "V", "dtype", "n_hist", "n_bias")] + \
        [(n, ctypes.c_int64) for n in ("ld", "ld_out", "ld_history", "ld_bias", "ld_allowed")]


def make_adjust(N, V, ld, dtype, n_hist=0, n_bias=0, ld_out=None, ld_history=None, ld_bias=None,
                ld_allowed=None):
    """Elements between the rows of each array: ld_out like ld, the others side by side if None."""
    return tfm_adjust.from_buffer_copy(_ADJUST.pack(
        N, V, _DTYPES.get(dtype, dtype), n_hist, n_bias, ld, ld if ld_out is None else ld_out,
        n_hist if ld_history is None else ld_history, n_bias if ld_bias is None else ld_bias,
        (V + 31) // 32 if ld_allowed is None else ld_allowed))


class tfm_cache8(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("heads", "d", "page", "n_pages")]


def make_cache8(heads, d, page, n_pages):
    return tfm_cache8(int(heads), int(d), int(page), int(n_pages))


class tfm_cache8_rows(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "L", "max_pages", "dtype")] + \
        [(n, ctypes.c_int64 * 3) for n in ("stride_k", "stride_v")]


def make_cache8_rows(B, L, max_pages, dtype, stride_k, stride_v):
    """stride_k, stride_v: elements between sequences, rows and heads."""
    if len(stride_k) != 3 or len(stride_v) != 3:
        raise ValueError(f"need three strides each, got {stride_k} and {stride_v}")
    return tfm_cache8_rows.from_buffer_copy(_ROWS.pack(
        B, L, max_pages, _DTYPES.get(dtype, dtype), *stride_k, *stride_v))


class tfm_cache8_query(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "L", "max_pages", "max_len", "heads", "causal",
                                               "dtype")] + [("scale", ctypes.c_float)] + \
        [(n, ctypes.c_int64 * 3) for n in ("stride_q", "stride_out")]


def make_cache8_query(B, L, heads, max_pages, dtype, stride_q, stride_out, scale, causal=False,
                      max_len=0):
    """stride_q, stride_out: elements between sequences, rows and heads; max_len: no sequence is
    longer (0: not said)."""
    if len(stride_q) != 3 or len(stride_out) != 3:
        raise ValueError(f"need three strides each, got {stride_q} and {stride_out}")
    return tfm_cache8_query.from_buffer_copy(_QUERY.pack(
        B, L, max_pages, max_len, heads, bool(causal), _DTYPES.get(dtype, dtype), scale, *stride_q,
        *stride_out))


def lib():
    """Loads the library (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                               "python paper_2606_03681_amd/build.py")
        L = ctypes.CDLL(_LIB_PATH)
        P = ctypes.POINTER
        vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
        for name in ("tfm_layer_param_count", "tfm_layer_saved_bytes",
                     "tfm_layer_workspace_bytes", "tfm_infer_workspace_bytes",
                     "tfm_infer_cache_bytes", "tfm_infer_cache8_bytes"):
            getattr(L, name).restype = sz
            getattr(L, name).argtypes = [P(tfm_dims)]
        L.tfm_last_error.restype = ctypes.c_char_p
        L.tfm_last_error.argtypes = []
        L.tfm_layer_fwd.restype = i32
        L.tfm_layer_fwd.argtypes = [P(tfm_dims), vp, vp, vp, vp, vp, vp, sz, vp, sz, vp]
        L.tfm_layer_fwd_noalloc.restype = i32
        L.tfm_layer_fwd_noalloc.argtypes = [P(tfm_dims), vp, vp, vp, vp, vp, vp, sz, vp]
        L.tfm_layer_bwd.restype = i32
        L.tfm_layer_bwd.argtypes = [P(tfm_dims), vp, vp, vp, vp, vp, sz, vp, vp, vp, i32, vp,
                                    sz, vp]
        L.tfm_thinking_rows_fwd.restype = i32
        L.tfm_thinking_rows_fwd.argtypes = [P(tfm_dims), vp, vp, i32, vp, vp, vp, sz, vp]
        L.tfm_thinking_rows_bwd.restype = i32
        L.tfm_thinking_rows_bwd.argtypes = [P(tfm_dims), vp, vp, i32, vp, vp, i32, vp, sz, vp]
        L.tfm_layer_fwd_context.restype = i32
        L.tfm_layer_fwd_context.argtypes = [P(tfm_dims), vp, vp, vp, vp, vp, vp, sz, vp, sz, vp]
        L.tfm_layer_fwd_query.restype = i32
        L.tfm_layer_fwd_query.argtypes = [P(tfm_dims), i32, vp, vp, vp, vp, vp, sz, vp, vp, sz,
                                          vp]
        L.tfm_infer8_workspace_bytes.restype = sz
        L.tfm_infer8_workspace_bytes.argtypes = [P(tfm_dims), i32]
        L.tfm_layer_fwd_context8.restype = i32
        L.tfm_layer_fwd_context8.argtypes = [P(tfm_dims), vp, vp, vp, vp, vp, vp, sz, vp, sz, vp,
                                             sz, vp]
        L.tfm_layer_fwd_query8.restype = i32
        L.tfm_layer_fwd_query8.argtypes = [P(tfm_dims), i32, vp, vp, vp, vp, vp, sz, vp, vp, sz,
                                           vp]
        E_ = P(tfm_ends)
        for name in ("tfm_ends_param_count", "tfm_ends_workspace_bytes"):
            getattr(L, name).restype = sz
            getattr(L, name).argtypes = [P(tfm_dims), E_]
        L.tfm_encode_fwd.restype = i32
        L.tfm_encode_fwd.argtypes = [P(tfm_dims), E_, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.tfm_encode_bwd.restype = i32
        L.tfm_encode_bwd.argtypes = [P(tfm_dims), E_, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
        L.tfm_decode_fwd.restype = i32
        L.tfm_decode_fwd.argtypes = [P(tfm_dims), E_, vp, vp, vp, vp, vp, vp, sz, vp]
        L.tfm_decode_loss.restype = i32
        L.tfm_decode_loss.argtypes = [P(tfm_dims), E_, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                      i32, vp, sz, vp]
        L.tfm_decode_bwd.restype = i32
        L.tfm_decode_bwd.argtypes = [P(tfm_dims), E_, vp, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
        L.tfm_embed_workspace_bytes.restype = sz
        L.tfm_embed_workspace_bytes.argtypes = [P(tfm_embed)]
        L.tfm_embed_fwd.restype = i32
        L.tfm_embed_fwd.argtypes = [P(tfm_embed), vp, vp, vp, i32, vp]
        L.tfm_embed_bwd.restype = i32
        L.tfm_embed_bwd.argtypes = [P(tfm_embed), vp, vp, vp, i32, vp, sz, vp]
        L.tfm_distill_workspace_bytes.restype = sz
        L.tfm_distill_workspace_bytes.argtypes = [P(tfm_distill)]
        L.tfm_distill_loss.restype = i32
        L.tfm_distill_loss.argtypes = [P(tfm_distill)] + [vp] * 11 + [sz, vp]
        L.tfm_sample.restype = i32
        L.tfm_sample.argtypes = [P(tfm_sampling)] + [vp] * 10
        L.tfm_adjust_logits.restype = i32
        L.tfm_adjust_logits.argtypes = [P(tfm_adjust)] + [vp] * 12
        C8 = P(tfm_cache8)
        L.tfm_cache8_bytes.restype = sz
        L.tfm_cache8_bytes.argtypes = [C8]
        L.tfm_cache8_append.restype = i32
        L.tfm_cache8_append.argtypes = [C8, P(tfm_cache8_rows)] + [vp] * 6 + [sz, vp]
        L.tfm_cache8_attend_workspace_bytes.restype = sz
        L.tfm_cache8_attend_workspace_bytes.argtypes = [C8, P(tfm_cache8_query)]
        L.tfm_cache8_attend.restype = i32
        L.tfm_cache8_attend.argtypes = [C8, P(tfm_cache8_query)] + [vp] * 5 + [sz] + [vp] * 3 + \
            [sz, vp]
        i64, f32 = ctypes.c_int64, ctypes.c_float
        L.tfm_clip_workspace_bytes.restype = sz
        L.tfm_clip_workspace_bytes.argtypes = [i32, P(i64)]
        L.tfm_clip_scale.restype = i32
        L.tfm_clip_scale.argtypes = [i32, P(vp), P(i64), f32, vp, vp, vp, sz, vp]
        L.tfm_sfadamw_step.restype = i32
        L.tfm_sfadamw_step.argtypes = [P(tfm_sfadamw), i64, i32, P(i64), P(i64), vp, vp, vp, vp,
                                       vp, vp]
        L.tfm_muon_workspace_bytes.restype = sz
        L.tfm_muon_workspace_bytes.argtypes = [i32, i32, i32]
        L.tfm_muon_step.restype = i32
        L.tfm_muon_step.argtypes = [P(tfm_muon), i32, i32, i32, P(vp), P(vp), P(vp), vp, vp, sz,
                                    vp]
        L.tfm_prof_enable.restype = i32
        L.tfm_prof_enable.argtypes = [i32]
        L.tfm_prof_collect.restype = i32
        L.tfm_prof_collect.argtypes = []
        L.tfm_prof_step.restype = i32
        L.tfm_prof_step.argtypes = [i32, P(ctypes.c_char_p), P(ctypes.c_longlong),
                                    P(ctypes.c_double)]
        L.tfm_prof_item_bwd_fused_rows.restype = i32
        L.tfm_prof_item_bwd_fused_rows.argtypes = [i32]
        L.tfm_prof_item_bwd_columns.restype = i32
        L.tfm_prof_item_bwd_columns.argtypes = [P(tfm_dims), vp, vp, vp]
        _lib = L
    return _lib


def last_error():
    return lib().tfm_last_error().decode()


def param_count(dims):
    return lib().tfm_layer_param_count(ctypes.byref(dims))


def saved_bytes(dims):
    return lib().tfm_layer_saved_bytes(ctypes.byref(dims))


def workspace_bytes(dims):
    return lib().tfm_layer_workspace_bytes(ctypes.byref(dims))


def infer_workspace_bytes(dims):
    return lib().tfm_infer_workspace_bytes(ctypes.byref(dims))


def infer_cache_bytes(dims):
    return lib().tfm_infer_cache_bytes(ctypes.byref(dims))


def infer_cache8_bytes(dims):
    return lib().tfm_infer_cache8_bytes(ctypes.byref(dims))


def infer8_workspace_bytes(dims, context_rows):
    return lib().tfm_infer8_workspace_bytes(ctypes.byref(dims), int(context_rows))


def _ptr(t):
    return t if t is None or isinstance(t, int) else t.data_ptr()


def _ptrs(*tensors):
    return [None if t is None else t.data_ptr() for t in tensors]


def _host(a, dtype):
    a = np.ascontiguousarray(a, dtype=dtype)
    return a, a.ctypes.data


def _check(rc):
    if rc != 0:
        raise TfmError(rc, last_error())


def _stream(stream):
    if stream is None:
        import torch
        # the handle itself, 0.3 us: torch.cuda.current_stream() takes 2.7 us to build a Stream, but
        # is the public way to it
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is None:
            return torch.cuda.current_stream().cuda_stream
        return raw(torch.cuda.current_device())
    return stream if isinstance(stream, int) else stream.cuda_stream


def layer_fwd(dims, n_train, cell_mask, X, params, Y, saved, workspace, stream=None):
    """tfm_layer_fwd.  n_train: host int32 [B]; cell_mask: host uint8 [B, C+1]; X, Y: device
    tensors [B, R, C+1, E] (float32 or bfloat16); params: device float32; saved, workspace:
    device byte tensors of saved_bytes(dims) / workspace_bytes(dims)."""
    nt, ntp = _host(n_train, np.int32)
    cm, cmp_ = _host(cell_mask, np.uint8)
    rc = lib().tfm_layer_fwd(ctypes.byref(dims), ntp, cmp_, _ptr(X), _ptr(params), _ptr(Y),
                             _ptr(saved), _nbytes(saved),
                             _ptr(workspace), _nbytes(workspace),
                             _stream(stream))
    _check(rc)


def layer_fwd_noalloc(dims, n_train, cell_mask, X, params, Y, saved, stream=None):
    """tfm_layer_fwd_noalloc: tfm_layer_fwd with its scratch in the library's own device array
    (no workspace argument; calls on one GPU must not overlap)."""
    nt, ntp = _host(n_train, np.int32)
    cm, cmp_ = _host(cell_mask, np.uint8)
    rc = lib().tfm_layer_fwd_noalloc(ctypes.byref(dims), ntp, cmp_, _ptr(X), _ptr(params),
                                     _ptr(Y), _ptr(saved), _nbytes(saved),
                                     _stream(stream))
    _check(rc)


def layer_bwd(dims, n_train, cell_mask, X, params, saved, dY, dX, grads, accumulate, workspace,
              stream=None):
    """tfm_layer_bwd; grads: device float32 like params, overwritten or accumulated."""
    nt, ntp = _host(n_train, np.int32)
    cm, cmp_ = _host(cell_mask, np.uint8)
    rc = lib().tfm_layer_bwd(ctypes.byref(dims), ntp, cmp_, _ptr(X), _ptr(params), _ptr(saved),
                             _nbytes(saved), _ptr(dY), _ptr(dX),
                             _ptr(grads), int(bool(accumulate)), _ptr(workspace),
                             _nbytes(workspace), _stream(stream))
    _check(rc)


def thinking_rows_fwd(dims, n_train, cell_mask, T, table, X, workspace, stream=None):
    """tfm_thinking_rows_fwd: writes table (device float32 [T, E]) into rows [0, T) of X
    (device [B, R, C+1, E]) at active columns, 0 at inactive ones."""
    nt, ntp = _host(n_train, np.int32)
    cm, cmp_ = _host(cell_mask, np.uint8)
    rc = lib().tfm_thinking_rows_fwd(ctypes.byref(dims), ntp, cmp_, int(T), _ptr(table), _ptr(X),
                                     _ptr(workspace),
                                     _nbytes(workspace),
                                     _stream(stream))
    _check(rc)


def thinking_rows_bwd(dims, n_train, cell_mask, T, dX, dtable, accumulate, workspace,
                      stream=None):
    """tfm_thinking_rows_bwd: dtable (device float32 [T, E]) gets (or adds) the sum of dX rows
    [0, T) over datasets and active columns."""
    nt, ntp = _host(n_train, np.int32)
    cm, cmp_ = _host(cell_mask, np.uint8)
    rc = lib().tfm_thinking_rows_bwd(ctypes.byref(dims), ntp, cmp_, int(T), _ptr(dX),
                                     _ptr(dtable), int(bool(accumulate)), _ptr(workspace),
                                     _nbytes(workspace),
                                     _stream(stream))
    _check(rc)


def _nbytes(t):
    """Bytes that the library may use from a buffer's first on."""
    if t is None:
        return 0
    if not t.is_contiguous():
        raise ValueError(f"a buffer of shape {tuple(t.shape)} and strides {t.stride()}: its elements "
                         "have to lie side by side")
    return t.nbytes


def layer_fwd_context(dims, n_train, cell_mask, X, params, Y, kv_cache, workspace, stream=None):
    """tfm_layer_fwd_context: forward without saved state; the train rows' item-axis keys and
    values go to kv_cache (a device byte tensor of infer_cache_bytes(dims))."""
    nt, ntp = _host(n_train, np.int32)
    cm, cmp_ = _host(cell_mask, np.uint8)
    rc = lib().tfm_layer_fwd_context(ctypes.byref(dims), ntp, cmp_, _ptr(X), _ptr(params),
                                     _ptr(Y), _ptr(kv_cache), _nbytes(kv_cache), _ptr(workspace),
                                     _nbytes(workspace), _stream(stream))
    _check(rc)


def layer_fwd_query(dims, context_rows, n_train, cell_mask, X, params, kv_cache, Y, workspace,
                    stream=None):
    """tfm_layer_fwd_query: forward of unlabelled rows X [B, Rq, C+1, E] against the keys and
    values a context call with context_rows rows left in kv_cache."""
    nt, ntp = _host(n_train, np.int32)
    cm, cmp_ = _host(cell_mask, np.uint8)
    rc = lib().tfm_layer_fwd_query(ctypes.byref(dims), int(context_rows), ntp, cmp_, _ptr(X),
                                   _ptr(params), _ptr(kv_cache), _nbytes(kv_cache), _ptr(Y),
                                   _ptr(workspace), _nbytes(workspace), _stream(stream))
    _check(rc)


def layer_fwd_context8(dims, n_train, cell_mask, X, params, Y, kv_cache, cache8, workspace,
                       stream=None):
    """tfm_layer_fwd_context8: the context call, with the train rows' keys and values kept in cache8
    (a device byte tensor of infer_cache8_bytes(dims)); kv_cache is scratch."""
    nt, ntp = _host(n_train, np.int32)
    cm, cmp_ = _host(cell_mask, np.uint8)
    rc = lib().tfm_layer_fwd_context8(ctypes.byref(dims), ntp, cmp_, _ptr(X), _ptr(params), _ptr(Y),
                                      _ptr(kv_cache), _nbytes(kv_cache), _ptr(cache8),
                                      _nbytes(cache8), _ptr(workspace), _nbytes(workspace),
                                      _stream(stream))
    _check(rc)


def layer_fwd_query8(dims, context_rows, n_train, cell_mask, X, params, cache8, Y, workspace,
                     stream=None):
    """tfm_layer_fwd_query8: the query call against the keys and values that a context8 call with
    context_rows rows left in cache8; workspace: infer8_workspace_bytes(dims, context_rows)."""
    nt, ntp = _host(n_train, np.int32)
    cm, cmp_ = _host(cell_mask, np.uint8)
    rc = lib().tfm_layer_fwd_query8(ctypes.byref(dims), int(context_rows), ntp, cmp_, _ptr(X),
                                    _ptr(params), _ptr(cache8), _nbytes(cache8), _ptr(Y),
                                    _ptr(workspace), _nbytes(workspace), _stream(stream))
    _check(rc)


def ends_param_count(dims, ends):
    return lib().tfm_ends_param_count(ctypes.byref(dims), ctypes.byref(ends))


def ends_workspace_bytes(dims, ends):
    return lib().tfm_ends_workspace_bytes(ctypes.byref(dims), ctypes.byref(ends))


def encode_fwd(dims, ends, n_train, n_feat, x, labels, params, X, workspace, stream=None):
    """tfm_encode_fwd.  n_train, n_feat: host int32 [B]; x: device float32 [B, R-T, F];
    labels: device int32 [B, R-T]; params: device float32 packed ends vector; X: device
    [B, R, C+1, E] (rows [T, R) written)."""
    nt, ntp = _host(n_train, np.int32)
    nf, nfp = _host(n_feat, np.int32)
    rc = lib().tfm_encode_fwd(ctypes.byref(dims), ctypes.byref(ends), ntp, nfp, _ptr(x),
                              _ptr(labels), _ptr(params), _ptr(X), _ptr(workspace),
                              _nbytes(workspace), _stream(stream))
    _check(rc)


def encode_bwd(dims, ends, n_train, n_feat, x, labels, dX, grads, accumulate, workspace,
               stream=None):
    """tfm_encode_bwd: the encoder entries of grads from dX (device [B, R, C+1, E])."""
    nt, ntp = _host(n_train, np.int32)
    nf, nfp = _host(n_feat, np.int32)
    rc = lib().tfm_encode_bwd(ctypes.byref(dims), ctypes.byref(ends), ntp, nfp, _ptr(x),
                              _ptr(labels), _ptr(dX), _ptr(grads), int(bool(accumulate)),
                              _ptr(workspace), _nbytes(workspace), _stream(stream))
    _check(rc)


def decode_fwd(dims, ends, n_train, n_feat, Y, params, logits, workspace, stream=None):
    """tfm_decode_fwd: logits (device float32 [T_test, K]) of the unlabelled rows of Y."""
    nt, ntp = _host(n_train, np.int32)
    nf, nfp = _host(n_feat, np.int32)
    rc = lib().tfm_decode_fwd(ctypes.byref(dims), ctypes.byref(ends), ntp, nfp, _ptr(Y),
                              _ptr(params), _ptr(logits), _ptr(workspace), _nbytes(workspace),
                              _stream(stream))
    _check(rc)


def decode_loss(dims, ends, n_train, n_feat, n_class, labels, Y, params, loss, logits, dY, grads,
                accumulate, workspace, stream=None):
    """tfm_decode_loss: loss (device float32 [1]), logits (device float32 [T_test, K] or None),
    dY (device like Y) and the decoder entries of grads."""
    nt, ntp = _host(n_train, np.int32)
    nf, nfp = _host(n_feat, np.int32)
    nc, ncp = _host(n_class, np.int32)
    rc = lib().tfm_decode_loss(ctypes.byref(dims), ctypes.byref(ends), ntp, nfp, ncp,
                               _ptr(labels), _ptr(Y), _ptr(params), _ptr(loss), _ptr(logits),
                               _ptr(dY), _ptr(grads), int(bool(accumulate)), _ptr(workspace),
                               _nbytes(workspace), _stream(stream))
    _check(rc)


def decode_bwd(dims, ends, n_train, n_feat, Y, params, dlogits, dY, grads, accumulate, workspace,
               stream=None):
    """tfm_decode_bwd: dY (device like Y) and the decoder entries of grads for the gradient dlogits
    (device float32 [T_test, K]) of decode_fwd's logits."""
    nt, ntp = _host(n_train, np.int32)
    nf, nfp = _host(n_feat, np.int32)
    rc = lib().tfm_decode_bwd(ctypes.byref(dims), ctypes.byref(ends), ntp, nfp, _ptr(Y),
                              _ptr(params), _ptr(dlogits), _ptr(dY), _ptr(grads),
                              int(bool(accumulate)), _ptr(workspace), _nbytes(workspace),
                              _stream(stream))
    _check(rc)


def _tensors(call, *wanted):
    """(name, tensor, type, shape) of a call's device tensors, None for one left out: raises unless
    every tensor has its type (None: any) and shape, lies side by side (shape None: not looked at)
    and all are on the current device."""
    import torch
    device = None
    for name, t, dtype, shape in wanted:
        if t is None:
            continue
        if dtype is not None and t.dtype is not dtype:
            raise ValueError(f"{call}: {name} is {t.dtype}, {dtype} wanted")
        if shape is not None and (t.shape != shape or not t.is_contiguous()):
            raise ValueError(f"{call}: {name} has shape {tuple(t.shape)} and strides {t.stride()}, "
                             f"{tuple(shape)} side by side wanted")
        at = t.get_device()  # -1 off the GPU
        if device is None:
            device = torch.cuda.current_device() if at >= 0 else -1
        if at != device or at < 0:
            raise ValueError(f"{call}: {name} is on {t.device}, not on the current GPU")


def _torch_dtype(dtype):
    import torch
    return torch.bfloat16 if dtype == TFM_BF16 else torch.float32


def _strided_rows(call, name, t, dtype, shape, stride, width):
    """Rows of `width` elements along three axes: from the first row on, room for the last."""
    (a, b, c), (x, y, z) = shape, stride
    last = (a - 1) * x + (b - 1) * y + (c - 1) * z + width
    room = t.untyped_storage().nbytes() // t.itemsize - t.storage_offset()
    if last > room and a and b and c:
        raise ValueError(f"{call}: {name} has room for {room} elements, {last} wanted")
    return name, t, dtype, None


def _embed_rows(call, e, name, t):
    """The activations of an embedding call."""
    return _strided_rows(call, name, t, _torch_dtype(e.dtype), e.n, e.stride, e.E)


def _side_rows(call, a, name, t, dtype, width, ld):
    """Rows of what goes with a row of logits, ld elements apart: room for the last."""
    if t is not None and a.N and width and not (t.shape == (a.N, width) and t.stride() == (ld, 1)):
        room = t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()
        if (a.N - 1) * ld + width > room:
            raise ValueError(f"{call}: {name} has room for {room} elements, "
                             f"{(a.N - 1) * ld + width} wanted")
        if t.stride(-1) != 1 and t.shape[-1] > 1:
            raise ValueError(f"{call}: the rows of {name} are {t.stride(-1)} elements a step")
        if t.dim() == 2 and 1 < a.N == t.shape[0] and t.stride(0) != ld:
            raise ValueError(f"{call}: the rows of {name} are {t.stride(0)} elements apart, "
                             f"{ld} wanted")
    return name, t, dtype, None


def _logit_rows(call, d, name, t, ld=None):
    """Rows of logits, ld elements apart."""
    if t is None:
        return name, t, None, None
    N, V = d.N, d.V
    ld = d.ld if ld is None else ld
    rows, step = t.stride() if t.dim() == 2 else (0, 0)
    if t.shape != (N, V) or (V > 1 and N and step != 1) or (N > 1 and rows != ld):
        raise ValueError(f"{call}: {name} has shape {tuple(t.shape)} and strides {t.stride()}, "
                         f"({N}, {V}) with rows {ld} apart wanted")
    return name, t, _torch_dtype(d.dtype), None


def embed_workspace_bytes(e):
    return lib().tfm_embed_workspace_bytes(ctypes.byref(e))


def embed_fwd(e, ids, table, out, accumulate=False, stream=None):
    """tfm_embed_fwd.  ids: device int32 of shape e.n; table: device [V, E]; out: device tensor
    whose first element is the first row's (rows e.stride apart)."""
    import torch
    _tensors("embed_fwd", ("ids", ids, torch.int32, tuple(e.n)),
             ("table", table, _torch_dtype(e.table_dtype), (e.V, e.E)),
             _embed_rows("embed_fwd", e, "out", out))
    rc = lib().tfm_embed_fwd(ctypes.byref(e), _ptr(ids), _ptr(table), _ptr(out),
                             int(bool(accumulate)), _stream(stream))
    _check(rc)


def embed_bwd(e, ids, dout, dtable, accumulate, workspace, stream=None):
    """tfm_embed_bwd: dtable (device float32 [V, E]) gets (or adds) the scaled sums of dout's rows
    by id; workspace: embed_workspace_bytes(e)."""
    import torch
    _tensors("embed_bwd", ("ids", ids, torch.int32, tuple(e.n)),
             _embed_rows("embed_bwd", e, "dout", dout),
             ("dtable", dtable, torch.float32, (e.V, e.E)),
             ("workspace", workspace, None, None))
    rc = lib().tfm_embed_bwd(ctypes.byref(e), _ptr(ids), _ptr(dout), _ptr(dtable),
                             int(bool(accumulate)), _ptr(workspace), _nbytes(workspace),
                             _stream(stream))
    _check(rc)


def distill_workspace_bytes(d):
    return lib().tfm_distill_workspace_bytes(ctypes.byref(d))


def distill_loss(d, logits, top_idx, top_logit, top_lse, labels, weights, n_class, loss, row_loss,
                 dlogits, workspace, stream=None):
    """tfm_distill_loss.  logits, dlogits: device [N, V], rows d.ld apart (dlogits None: loss
    alone; logits itself: in place); top_idx int32, top_logit float32 [N, k]; top_lse float32 [N]
    (tail); labels int32 [N] (alpha < 1); weights float32 [N], n_class int32 [N], row_loss float32
    [N] or None; loss: device float32, its first element is written."""
    import torch
    i32, f32 = torch.int32, torch.float32
    _tensors("distill_loss", _logit_rows("distill_loss", d, "logits", logits),
             _logit_rows("distill_loss", d, "dlogits", dlogits),
             ("top_idx", top_idx, i32, (d.N, d.k)), ("top_logit", top_logit, f32, (d.N, d.k)),
             ("top_lse", top_lse, f32, (d.N,)), ("labels", labels, i32, (d.N,)),
             ("weights", weights, f32, (d.N,)), ("n_class", n_class, i32, (d.N,)),
             ("loss", loss, f32, None), ("row_loss", row_loss, f32, (d.N,)),
             ("workspace", workspace, None, None))
    rc = lib().tfm_distill_loss(ctypes.byref(d), _ptr(logits), _ptr(top_idx), _ptr(top_logit),
                                _ptr(top_lse), _ptr(labels), _ptr(weights), _ptr(n_class),
                                _ptr(loss), _ptr(row_loss), _ptr(dlogits), _ptr(workspace),
                                _nbytes(workspace), _stream(stream))
    _check(rc)


def sample(s, logits, n_class, temperature, top_k, top_p, min_p, u, token, logprob=None,
           stream=None):
    """tfm_sample.  logits: device [N, V], rows s.ld apart; n_class, top_k int32 [N],
    temperature, top_p, min_p float32 [N], each or None; u float32 [N]; token int32 [N]; logprob
    float32 [N] or None."""
    import torch
    i32, f32, N = torch.int32, torch.float32, (s.N,)
    _tensors("sample", _logit_rows("sample", s, "logits", logits), ("n_class", n_class, i32, N),
             ("temperature", temperature, f32, N), ("top_k", top_k, i32, N),
             ("top_p", top_p, f32, N), ("min_p", min_p, f32, N), ("u", u, f32, N),
             ("token", token, i32, N), ("logprob", logprob, f32, N))
    rc = lib().tfm_sample(ctypes.byref(s), _ptr(logits), _ptr(n_class), _ptr(temperature),
                          _ptr(top_k), _ptr(top_p), _ptr(min_p), _ptr(u), _ptr(token),
                          _ptr(logprob), _stream(stream))
    _check(rc)


def adjust_logits(a, logits, n_class, history, n_history, repetition, presence, frequency,
                  bias_idx, bias, allowed, out, stream=None):
    """tfm_adjust_logits.  logits, out: device [N, V], rows a.ld and a.ld_out apart (out may be
    logits); n_class, n_history int32 [N], repetition, presence, frequency float32 [N], each or None;
    history int32, bias_idx int32, bias float32 and allowed int32 (bits): first elements of rows
    a.ld_history, a.ld_bias and a.ld_allowed apart, each or None."""
    import torch
    i32, f32, N = torch.int32, torch.float32, (a.N,)
    call = "adjust_logits"
    _tensors(call, _logit_rows(call, a, "logits", logits),
             _logit_rows(call, a, "out", out, a.ld_out), ("n_class", n_class, i32, N),
             _side_rows(call, a, "history", history, i32, a.n_hist, a.ld_history),
             ("n_history", n_history, i32, N), ("repetition", repetition, f32, N),
             ("presence", presence, f32, N), ("frequency", frequency, f32, N),
             _side_rows(call, a, "bias_idx", bias_idx, i32, a.n_bias, a.ld_bias),
             _side_rows(call, a, "bias", bias, f32, a.n_bias, a.ld_bias),
             _side_rows(call, a, "allowed", allowed, i32, (a.V + 31) // 32, a.ld_allowed))
    rc = lib().tfm_adjust_logits(
        ctypes.byref(a), *_ptrs(logits, n_class, history, n_history, repetition, presence,
                                frequency, bias_idx, bias, allowed, out), _stream(stream))
    _check(rc)


def cache8_bytes(c):
    return lib().tfm_cache8_bytes(ctypes.byref(c))


def cache8_views(c, pool):
    """The keys [n_pages, heads, page, d], values [n_pages, heads, d, page] (e4m3 codes) and powers
    [n_pages, heads, 2] (bytes e of 2^(e - 127)) of a pool, as views of it."""
    import torch
    n, h, d, p = c.n_pages, c.heads, c.d, c.page
    half, f8 = n * h * d * p, torch.float8_e4m3fn
    return (pool[:half].view(f8).view(n, h, p, d), pool[half:2 * half].view(f8).view(n, h, d, p),
            pool[2 * half:2 * half + 2 * n * h].view(n, h, 2))


def cache8_append(c, r, k, v, pages, lens, n_new, pool, stream=None):
    """tfm_cache8_append.  k, v: device tensors whose first elements are the first rows' (rows
    r.stride_k and r.stride_v apart); pages int32 [B, max_pages], lens, n_new int32 [B], each or
    None; pool: device bytes, cache8_bytes(c) of them."""
    import torch
    i32, n, dtype = torch.int32, (r.B, r.L, c.heads), _torch_dtype(r.dtype)
    _tensors("cache8_append", _strided_rows("cache8_append", "k", k, dtype, n, r.stride_k, c.d),
             _strided_rows("cache8_append", "v", v, dtype, n, r.stride_v, c.d),
             ("pages", pages, i32, (r.B, r.max_pages)), ("lens", lens, i32, (r.B,)),
             ("n_new", n_new, i32, (r.B,)), ("pool", pool, None, None))
    rc = lib().tfm_cache8_append(ctypes.byref(c), ctypes.byref(r),
                                 *_ptrs(k, v, pages, lens, n_new, pool), _nbytes(pool),
                                 _stream(stream))
    _check(rc)


def cache8_attend_workspace_bytes(c, a):
    return lib().tfm_cache8_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(a))


def cache8_attend(c, a, q, pages, lens, n_rows, pool, out, lse, workspace, stream=None):
    """tfm_cache8_attend.  q, out: device tensors whose first elements are the first rows' (rows
    a.stride_q and a.stride_out apart); pages int32 [B, max_pages] or None; lens int32 [B]; n_rows
    int32 [B] or None; lse float32 [B, L, heads] or None; workspace: device bytes,
    cache8_attend_workspace_bytes(c, a) of them (None for 0)."""
    import torch
    i32, n, dtype = torch.int32, (a.B, a.L, a.heads), _torch_dtype(a.dtype)
    _tensors("cache8_attend", _strided_rows("cache8_attend", "q", q, dtype, n, a.stride_q, c.d),
             _strided_rows("cache8_attend", "out", out, dtype, n, a.stride_out, c.d),
             ("pages", pages, i32, (a.B, a.max_pages)), ("lens", lens, i32, (a.B,)),
             ("n_rows", n_rows, i32, (a.B,)), ("pool", pool, None, None),
             ("lse", lse, torch.float32, n), ("workspace", workspace, None, None))
    rc = lib().tfm_cache8_attend(ctypes.byref(c), ctypes.byref(a),
                                 *_ptrs(q, pages, lens, n_rows, pool), _nbytes(pool),
                                 *_ptrs(out, lse, workspace), _nbytes(workspace), _stream(stream))
    _check(rc)


def _ptr_array(ptrs):
    return (ctypes.c_void_p * len(ptrs))(*[int(p) for p in ptrs])


def _i64_array(vals):
    return (ctypes.c_int64 * len(vals))(*[int(v) for v in vals])


def clip_workspace_bytes(counts):
    return lib().tfm_clip_workspace_bytes(len(counts), _i64_array(counts))


def clip_scale(grads, max_norm, scale, norm, workspace, stream=None):
    """tfm_clip_scale over device float32 tensors (or (pointer, count) pairs): writes the clip
    factor to scale[0] and the global norm to norm[0] (norm may be None)."""
    ptrs = [g[0] if isinstance(g, tuple) else g.data_ptr() for g in grads]
    counts = [g[1] if isinstance(g, tuple) else g.numel() for g in grads]
    rc = lib().tfm_clip_scale(len(ptrs), _ptr_array(ptrs), _i64_array(counts), float(max_norm),
                              _ptr(scale), _ptr(norm), _ptr(workspace), _nbytes(workspace),
                              _stream(stream))
    _check(rc)


def sfadamw_step(hp, t, segments, y, z, v, grad, grad_scale=None, stream=None):
    """tfm_sfadamw_step; segments: list of (offset, length) into the float32 vectors."""
    offs = [o for o, _ in segments]
    lens = [n for _, n in segments]
    rc = lib().tfm_sfadamw_step(ctypes.byref(hp), int(t), len(segments), _i64_array(offs),
                                _i64_array(lens), _ptr(y), _ptr(z), _ptr(v), _ptr(grad),
                                _ptr(grad_scale), _stream(stream))
    _check(rc)


def muon_workspace_bytes(count, rows, cols):
    return lib().tfm_muon_workspace_bytes(int(count), int(rows), int(cols))


def muon_step(hp, rows, cols, W, G, buf, grad_scale, workspace, stream=None):
    """tfm_muon_step on len(W) matrices of rows x cols; W, G, buf: lists of device pointers (or
    tensors) of the same length."""
    conv = [[p if isinstance(p, int) else p.data_ptr() for p in lst] for lst in (W, G, buf)]
    rc = lib().tfm_muon_step(ctypes.byref(hp), len(conv[0]), int(rows), int(cols),
                             _ptr_array(conv[0]), _ptr_array(conv[1]), _ptr_array(conv[2]),
                             _ptr(grad_scale), _ptr(workspace), _nbytes(workspace),
                             _stream(stream))
    _check(rc)


def prof_enable(on=True):
    """Turns per-step HIP-event timing of the library's launches on or off (tfm_prof.h)."""
    _check(lib().tfm_prof_enable(int(bool(on))))


def prof_item_bwd_fused_rows(head_dim):
    """Longest train prefix whose item-attention backward runs as the one-kernel step
    "item_attn_bwd" at this head dimension (0: never); see tfm_prof.h."""
    return int(lib().tfm_prof_item_bwd_fused_rows(int(head_dim)))


def prof_item_bwd_columns(dims, n_train, cell_mask):
    """(number of columns of the one-kernel item-attention backward, every active column in launch
    order) for a backward call; see tfm_prof.h."""
    n = np.ascontiguousarray(n_train, dtype=np.int32)
    m = np.ascontiguousarray(cell_mask, dtype=np.uint8)
    order = np.empty(int(np.count_nonzero(m)), np.int32)
    k = lib().tfm_prof_item_bwd_columns(ctypes.byref(dims), n.ctypes.data, m.ctypes.data,
                                        order.ctypes.data)
    if k < 0:
        raise TfmError(k, last_error())
    return k, order


def prof_collect():
    """Waits for the recorded events; returns {step: (launches, total_ms)}."""
    n = lib().tfm_prof_collect()
    if n < 0:
        raise TfmError(n, "profiling events could not be read")
    out = {}
    for i in range(n):
        name = ctypes.c_char_p()
        cnt = ctypes.c_longlong()
        ms = ctypes.c_double()
        lib().tfm_prof_step(i, ctypes.byref(name), ctypes.byref(cnt), ctypes.byref(ms))
        out[name.value.decode()] = (cnt.value, ms.value)
    return out
