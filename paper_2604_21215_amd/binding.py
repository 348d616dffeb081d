"""ctypes binding of librt_hip.so: the same entry points as include/rt.h, argument marshalling only.

Every step of the layer runs in the library's HIP kernels; PyTorch is used by callers for device
memory and streams.  There is no CPU fallback: if the library is missing the import of the symbols
fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os
import sys as _sys

from . import build as _build

RT_OK = 0
RT_ERR_INVALID_ARG, RT_ERR_UNSUPPORTED, RT_ERR_OOM, RT_ERR_HIP, RT_ERR_STATE = 1, 2, 3, 4, 5
RT_F32, RT_BF16 = 0, 1
RT_FLAG_NORM_FREE = 0x1
RT_FLAG_ENGINE_STEPWISE = 0x2
RT_FLAG_ENGINE_PERSISTENT = 0x4
RT_FLAG_NO_MFMA = 0x8
RT_FLAG_HIP_GRAPH = 0x10
RT_FLAG_DEBUG_POISON = 0x20
RT_RESERVE_LOOP_FREE, RT_RESERVE_BACKWARD, RT_RESERVE_PAGED = 0x1, 0x2, 0x4

EXPORTS = ("rt_create", "rt_layer_prefill", "rt_decode_step", "rt_destroy", "rt_last_error", "rt_status_string",
           "rt_workspace_bytes", "rt_device_wait_expired", "rt_engine_name", "rt_engine_form", "rt_schedule_events", "rt_partial_slot",
           "rt_version", "rt_phase_trace", "rt_schedule_events_shifted", "rt_embed_rows", "rt_lm_head", "rt_cross_block_event",
           "rt_stack_prefill", "rt_schedule_events_chunked", "rt_layer_recompute", "rt_transformer_layer",
           "rt_layer_prefill_blocked", "rt_decode_step_static", "rt_layer_backward", "rt_decode_phase_trace",
           "rt_cache_write", "rt_cache_read", "rt_paged_attention", "rt_decode_step_paged", "rt_mx4_pack", "rt_lm_head_mx4")


class rt_config(C.Structure):
    _fields_ = [
        ("d_model", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32), ("d_hidden", C.c_int32),
        ("max_batch", C.c_int32), ("max_seq", C.c_int32), ("dtype", C.c_int32), ("p_min", C.c_int32),
        ("resid_scale", C.c_float), ("attn_scale", C.c_float), ("rms_eps", C.c_float), ("flags", C.c_uint32),
        ("device", C.c_int32), ("stream", C.c_void_p), ("alibi_max_bias", C.c_float),
        ("reserve_stack_layers", C.c_int32), ("reserve_stack_chunk", C.c_int32), ("reserve", C.c_uint32),
    ]


class rt_layer_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("Wq", "Wk", "Wv", "Wo", "W1", "W2", "g_attn", "g_mlp", "g_kv", "g_q", "g_k")]


class rt_layer_grads(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("Wq", "Wk", "Wv", "Wo", "W1", "W2", "g_attn", "g_mlp", "g_kv", "g_q", "g_k")]


class rt_paged_cache(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("K_exp", C.c_void_p), ("V_exp", C.c_void_p), ("table", C.c_void_p),
                ("table_stride", C.c_int64), ("pages", C.c_int32), ("page_len", C.c_int32), ("bits", C.c_int32)]
    # set by make_cache: heads, bytes of an element and device in one number (0: not known), and the table's lines
    fit = 0, 1 << 31


class RTError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__("%s: %s" % (status, msg))
        self.status = status


_lib = None


def load():
    """Load the built library (builds it only if no library is there at all)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB):
        _build.build_hip(True)
    try:
        # callers hold their device memory in torch tensors: load torch's HIP runtime first so that the library binds
        # to the same one whatever the import order (two runtimes in one process do not share a device context)
        import torch  # noqa: F401
    except ImportError:
        pass
    L = C.CDLL(_build.LIB)
    ctxp = C.c_void_p
    L.rt_create.argtypes = [C.POINTER(rt_config), C.POINTER(ctxp)]
    L.rt_create.restype = C.c_int
    L.rt_layer_prefill.argtypes = [ctxp, C.POINTER(rt_layer_weights), C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                   C.c_void_p, C.c_void_p, C.c_int32]
    L.rt_layer_prefill.restype = C.c_int
    L.rt_decode_step.argtypes = [ctxp, C.POINTER(rt_layer_weights), C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                 C.c_void_p, C.c_void_p, C.c_int32]
    L.rt_decode_step.restype = C.c_int
    L.rt_destroy.argtypes = [ctxp]
    L.rt_destroy.restype = C.c_int
    L.rt_last_error.argtypes = [ctxp]
    L.rt_last_error.restype = C.c_char_p
    L.rt_status_string.argtypes = [C.c_int]
    L.rt_status_string.restype = C.c_char_p
    L.rt_workspace_bytes.argtypes = [ctxp]
    L.rt_workspace_bytes.restype = C.c_uint64
    L.rt_device_wait_expired.argtypes = [ctxp]
    L.rt_device_wait_expired.restype = C.c_int32
    L.rt_engine_name.argtypes = [ctxp]
    L.rt_engine_name.restype = C.c_char_p
    L.rt_engine_form.argtypes = [ctxp]
    L.rt_engine_form.restype = C.c_char_p
    L.rt_schedule_events.argtypes = [C.c_int32, C.c_int32, C.POINTER(C.c_int32), C.c_int32]
    L.rt_schedule_events.restype = C.c_int32
    L.rt_schedule_events_shifted.argtypes = [C.c_int32, C.c_int32, C.POINTER(C.c_int32), C.c_int32]
    L.rt_schedule_events_shifted.restype = C.c_int32
    L.rt_schedule_events_chunked.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_int32), C.c_int32]
    L.rt_schedule_events_chunked.restype = C.c_int32
    L.rt_partial_slot.argtypes = [C.c_int32, C.c_int32]
    L.rt_partial_slot.restype = C.c_int64
    L.rt_version.restype = C.c_int32
    L.rt_phase_trace.argtypes = [ctxp, C.POINTER(C.c_uint64), C.c_int32]
    L.rt_phase_trace.restype = C.c_int32
    L.rt_decode_phase_trace.argtypes = [ctxp, C.POINTER(C.c_uint64), C.c_int32]
    L.rt_decode_phase_trace.restype = C.c_int32
    L.rt_embed_rows.argtypes = [ctxp, C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_int32,
                                C.c_void_p]
    L.rt_embed_rows.restype = C.c_int
    L.rt_lm_head.argtypes = [ctxp, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p]
    L.rt_lm_head.restype = C.c_int
    L.rt_cross_block_event.argtypes = [ctxp, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32]
    L.rt_cross_block_event.restype = C.c_int
    L.rt_stack_prefill.argtypes = [ctxp, C.POINTER(rt_layer_weights), C.c_int32, C.c_void_p, C.c_int32, C.c_int32,
                                   C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.c_int32, C.c_int32]
    L.rt_stack_prefill.restype = C.c_int
    L.rt_layer_recompute.argtypes = [ctxp, C.POINTER(rt_layer_weights), C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32]
    L.rt_layer_recompute.restype = C.c_int
    L.rt_transformer_layer.argtypes = [ctxp, C.POINTER(rt_layer_weights), C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                       C.c_void_p, C.c_void_p, C.c_int32]
    L.rt_transformer_layer.restype = C.c_int
    L.rt_layer_prefill_blocked.argtypes = [ctxp, C.POINTER(rt_layer_weights), C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32]
    L.rt_layer_prefill_blocked.restype = C.c_int
    L.rt_decode_step_static.argtypes = [C.POINTER(rt_config), C.POINTER(rt_layer_weights), C.c_void_p, C.c_int32, C.c_int32,
                                        C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32]
    L.rt_decode_step_static.restype = C.c_int
    L.rt_layer_backward.argtypes = [ctxp, C.POINTER(rt_layer_weights), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.POINTER(rt_layer_grads)]
    L.rt_layer_backward.restype = C.c_int
    cachep = C.POINTER(rt_paged_cache)
    for fn in (L.rt_cache_write, L.rt_cache_read):
        fn.argtypes = [ctxp, cachep, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int64, C.c_int64]
        fn.restype = C.c_int
    L.rt_paged_attention.argtypes = [ctxp, cachep, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                     C.c_int64, C.c_void_p, C.c_int64, C.c_void_p]
    L.rt_paged_attention.restype = C.c_int
    L.rt_decode_step_paged.argtypes = [ctxp, C.POINTER(rt_layer_weights), cachep, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p]
    L.rt_decode_step_paged.restype = C.c_int
    L.rt_mx4_pack.argtypes = [C.c_void_p, C.c_int32, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p]
    L.rt_mx4_pack.restype = C.c_int
    L.rt_lm_head_mx4.argtypes = [ctxp, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p]
    L.rt_lm_head_mx4.restype = C.c_int
    _lib = L
    return L


def _check(L, ctx, rc):
    if rc != RT_OK:
        msg = L.rt_last_error(ctx).decode() if ctx else ""
        raise RTError(L.rt_status_string(rc).decode(), msg)


def _ptr(t):
    return C.c_void_p(0 if t is None else t.data_ptr())


def rt_decode_step_static(cfg: rt_config, weights: rt_layer_weights, x_t, t, y_t, K, V):
    """rt_decode_step_static(cfg, w, x_t[B,d], B, t, y_t, K, V, kv_cap): the decoding step without a context."""
    L = load()
    rc = L.rt_decode_step_static(C.byref(cfg), C.byref(weights), _ptr(x_t), x_t.shape[0], int(t), _ptr(y_t), _ptr(K), _ptr(V),
                                 K.shape[0])
    if rc != RT_OK:
        raise RTError(L.rt_status_string(rc).decode(), L.rt_last_error(None).decode())


def raw_decode_static(cfg, weights, x_ptr, B, t, y_ptr, K_ptr, V_ptr, kv_cap) -> int:
    """Status code of rt_decode_step_static on raw addresses (error-path tests)."""
    return load().rt_decode_step_static(C.byref(cfg), C.byref(weights), C.c_void_p(x_ptr), B, t, C.c_void_p(y_ptr),
                                        C.c_void_p(K_ptr), C.c_void_p(V_ptr), kv_cap)


def make_weights(w: dict) -> rt_layer_weights:
    """w maps names to device tensors (or None for the optional gains)."""
    s = rt_layer_weights()
    for name, _ in rt_layer_weights._fields_:
        t = w.get(name)
        setattr(s, name, None if t is None else t.data_ptr())
    return s


_INTS = "lengths, positions and counts are contiguous int32 on the context's device, one for each sequence"


def _invalid(msg):
    raise RTError("RT_ERR_INVALID_ARG", msg)


_dtypes = None


def _load_dtypes():   # an import statement in a call costs as much as three of its checks
    global _dtypes
    import torch
    _dtypes = torch.int8, torch.uint8, torch.int32, {torch.int8: 1, torch.bfloat16: 2, torch.float32: 4}
    return _dtypes


def _fit(heads, size, device):
    return heads << 16 | size << 12 | device + 2


def make_cache(K, V, table, K_exp=None, V_exp=None) -> rt_paged_cache:
    """K, V [pages, H, page_len, 64] (storage dtype, or int8 with the bytes K_exp, V_exp [pages, H, page_len]), table int32 [S, entries],
    contiguous: the kernels read whole lines, and follow any entry that a position leads to."""
    int8, uint8, int32, sizes = _dtypes or _load_dtypes()
    shape, dt, dev, ke, ve = K.shape, K.dtype, K.get_device(), None, None
    pages, heads, page_len, width = shape if len(shape) == 4 else (0, 0, 0, 0)
    if width != 64 or V.shape != shape or V.dtype is not dt or dt not in sizes or not (K.is_contiguous() and V.is_contiguous()):
        _invalid("K, V are contiguous [pages, H, page_len, 64] of one type: bfloat16, float32 or int8")
    if dt is int8 or K_exp is not None or V_exp is not None:
        if K_exp is None or V_exp is None or dt is not int8:
            _invalid("K_exp, V_exp belong to a cache of 8 bits (K, V int8), and to no other")
        for t in (K_exp, V_exp):
            if t.dtype is not uint8 or t.shape != shape[:3] or not t.is_contiguous() or t.get_device() != dev:
                _invalid("K_exp, V_exp are contiguous uint8 [pages, H, page_len] on the device of K")
        ke, ve = K_exp.data_ptr(), V_exp.data_ptr()
    lines, entries = table.shape
    if table.dtype is not int32 or not table.is_contiguous():   # a line's entries are all that lie up to the next line
        _invalid("table is contiguous int32 [S, entries]")
    if V.get_device() != dev or table.get_device() != dev:
        _invalid("K, V and table lie on one device")
    size = sizes[dt]
    c = rt_paged_cache(K.data_ptr(), V.data_ptr(), ke, ve, table.data_ptr(), entries, pages, page_len, 8 if size == 1 else 0)
    c.fit = heads << 16 | size << 12 | dev + 2, lines
    return c


def _pair_strides(k, v, H):
    """k, v [S, N, H, 64] with the same strides and the last two dimensions contiguous, dimensions of one row apart, which have no stride."""
    if len(k.shape) == 4 and v.shape == k.shape and tuple(k.shape[2:]) == (H, 64):
        S, N = k.shape[:2]
        strides = lambda t: (t.stride(0) if S > 1 else 0, t.stride(1) if N > 1 else 0, t.stride(2) if H > 1 else 64, t.stride(3))  # noqa: E731
        if strides(v) == strides(k) and strides(k)[2:] == (64, 1):
            return strides(k)[:2]
    _invalid("k and v are [S, N, n_heads, 64] with equal strides and contiguous heads")


def rt_mx4_pack(W):
    """W [rows, cols] on the host (numpy float32, or uint16 bf16 bits) -> (codes [rows, cols / 2], exps [rows, cols / 32]) uint8."""
    import numpy as np
    W = np.ascontiguousarray(W)
    if W.ndim != 2 or W.dtype not in (np.float32, np.uint16):
        raise RTError("RT_ERR_INVALID_ARG", "W is [rows, cols] float32 or uint16 (bf16 bits)")
    rows, cols = W.shape
    codes, exps = np.empty((rows, cols // 2), dtype=np.uint8), np.empty((rows, max(cols // 32, 1)), dtype=np.uint8)
    L = load()
    rc = L.rt_mx4_pack(W.ctypes.data, RT_F32 if W.dtype == np.float32 else RT_BF16, rows, cols, codes.ctypes.data, exps.ctypes.data)
    if rc != RT_OK:
        raise RTError(L.rt_status_string(rc).decode(), "rt_mx4_pack: cols a multiple of 32 and finite weights are required")
    return codes, exps


def _events(fn, N, p_min):
    n = fn(N, p_min, None, 0)
    if n < 0:
        raise RTError("RT_ERR_INVALID_ARG", "schedule")
    buf = (C.c_int32 * (5 * max(n, 1)))()
    fn(N, p_min, buf, n)
    return [tuple(buf[5 * i + j] for j in range(5)) for i in range(n)]


def rt_schedule_events(N: int, p_min: int):
    return _events(load().rt_schedule_events, N, p_min)


def rt_schedule_events_shifted(N: int, p_min: int):
    return _events(load().rt_schedule_events_shifted, N, p_min)


def rt_schedule_events_chunked(N: int, p_min: int, chunk: int):
    fn = load().rt_schedule_events_chunked
    return _events(lambda n, p, buf, cap: fn(n, p, chunk, buf, cap), N, p_min)


def rt_partial_slot(level: int, query: int) -> int:
    return int(load().rt_partial_slot(level, query))


class RTContext:
    """Owns an rt_ctx.  Methods mirror the C entry points and take torch device tensors."""

    def __init__(self, d_model, n_heads, d_hidden, max_batch, max_seq, dtype, *, p_min=0, resid_scale=1.0,
                 attn_scale=1.0, rms_eps=1e-6, flags=0, device=0, stream=None, alibi_max_bias=0.0, reserve_stack_layers=0,
                 reserve_stack_chunk=0, reserve=0):
        L = load()
        cfg = rt_config(d_model, n_heads, d_model // n_heads if n_heads else 0, d_hidden, max_batch, max_seq,
                        RT_BF16 if dtype in ("bf16", RT_BF16) and dtype != 0 else RT_F32, p_min, resid_scale, attn_scale,
                        rms_eps, flags, device, stream, alibi_max_bias, reserve_stack_layers, reserve_stack_chunk, reserve)
        self.cfg = cfg
        self._L = L
        self._ctx = C.c_void_p()
        rc = L.rt_create(C.byref(cfg), C.byref(self._ctx))
        if rc != RT_OK:
            raise RTError(L.rt_status_string(rc).decode(), "rt_create")

    # -- rt_layer_prefill(ctx, w, x[B,N,d], B, N, y, K, V, kv_cap)
    def rt_layer_prefill(self, weights: rt_layer_weights, x, y, K, V):
        B, N, _ = x.shape
        rc = self._L.rt_layer_prefill(self._ctx, C.byref(weights), _ptr(x), B, N, _ptr(y), _ptr(K), _ptr(V), K.shape[0])
        _check(self._L, self._ctx, rc)

    # -- rt_stack_prefill(ctx, layers[L], L, x[B,N,d], B, N, y[L], K[L], V[L], kv_cap, chunk)
    def rt_stack_prefill(self, weights: list, x, ys: list, Ks: list, Vs: list, chunk: int = 0):
        B, N, _ = x.shape
        L = len(weights)
        warr = (rt_layer_weights * L)(*weights)
        parr = lambda ts: (C.c_void_p * L)(*[t.data_ptr() for t in ts])
        rc = self._L.rt_stack_prefill(self._ctx, warr, L, _ptr(x), B, N, parr(ys), parr(Ks), parr(Vs), Ks[0].shape[0],
                                      int(chunk))
        _check(self._L, self._ctx, rc)

    def raw_stack_prefill(self, weights: list, x_ptr, B, N, y_ptrs, K_ptrs, V_ptrs, kv_cap, chunk) -> int:
        """Status code of rt_stack_prefill on raw addresses (error-path tests)."""
        L = len(weights)
        warr = (rt_layer_weights * L)(*weights)
        parr = lambda ps: (C.c_void_p * L)(*ps)
        return self._L.rt_stack_prefill(self._ctx, warr, L, C.c_void_p(x_ptr), B, N, parr(y_ptrs), parr(K_ptrs),
                                        parr(V_ptrs), kv_cap, chunk)

    # -- rt_layer_recompute(ctx, w, x[B,N,d], z[B,N,d], B, N, y, K, V, kv_cap)
    def rt_layer_recompute(self, weights: rt_layer_weights, x, z, y, K, V):
        B, N, _ = x.shape
        rc = self._L.rt_layer_recompute(self._ctx, C.byref(weights), _ptr(x), _ptr(z), B, N, _ptr(y), _ptr(K), _ptr(V),
                                        K.shape[0])
        _check(self._L, self._ctx, rc)

    # -- rt_layer_backward(ctx, w, x[B,N,d], z[B,N,d], gy[B,N,d], gK | None, gV | None, B, N, dx[B,N,d] f32, grads)
    def rt_layer_backward(self, weights: rt_layer_weights, x, z, gy, gK, gV, dx, grads: dict):
        """grads: name -> fp32 device tensor (any subset of the six matrices and five gains)."""
        B, N, _ = x.shape
        g = rt_layer_grads()
        for name, _t in rt_layer_grads._fields_:
            t = grads.get(name)
            setattr(g, name, None if t is None else t.data_ptr())
        rc = self._L.rt_layer_backward(self._ctx, C.byref(weights), _ptr(x), _ptr(z), _ptr(gy), _ptr(gK), _ptr(gV), B, N,
                                       _ptr(dx), C.byref(g))
        _check(self._L, self._ctx, rc)

    # -- rt_layer_prefill_blocked(ctx, w, x[B,N,d], B, N, block, y, K, V, kv_cap)
    def rt_layer_prefill_blocked(self, weights: rt_layer_weights, x, block, y, K, V):
        B, N, _ = x.shape
        rc = self._L.rt_layer_prefill_blocked(self._ctx, C.byref(weights), _ptr(x), B, N, int(block), _ptr(y), _ptr(K),
                                              _ptr(V), K.shape[0])
        _check(self._L, self._ctx, rc)

    # -- rt_transformer_layer(ctx, w, x[B,N,d], B, N, y, K, V, kv_cap)
    def rt_transformer_layer(self, weights: rt_layer_weights, x, y, K, V):
        B, N, _ = x.shape
        rc = self._L.rt_transformer_layer(self._ctx, C.byref(weights), _ptr(x), B, N, _ptr(y), _ptr(K), _ptr(V), K.shape[0])
        _check(self._L, self._ctx, rc)

    # -- rt_decode_step(ctx, w, x_t[B,d], B, t, y_t, K, V, kv_cap)
    def rt_decode_step(self, weights: rt_layer_weights, x_t, t, y_t, K, V):
        rc = self._L.rt_decode_step(self._ctx, C.byref(weights), _ptr(x_t), x_t.shape[0], int(t), _ptr(y_t), _ptr(K),
                                    _ptr(V), K.shape[0])
        _check(self._L, self._ctx, rc)

    # -- rt_embed_rows(ctx, table[vocab,d], vocab, ids[B,ids_stride] int32, ids_stride, first, B, N, x[B,N,d])
    def rt_embed_rows(self, table, ids, first, x):
        B, N, _ = x.shape
        rc = self._L.rt_embed_rows(self._ctx, _ptr(table), table.shape[0], _ptr(ids), ids.stride(0), int(first), B, N,
                                   _ptr(x))
        _check(self._L, self._ctx, rc)

    # -- rt_lm_head(ctx, W_lm[vocab,d], g_final[d] | None, vocab, z rows (stride z_stride elements), z_stride, B, logits[B,vocab] f32)
    def rt_lm_head(self, W_lm, g_final, z, z_stride, B, logits):
        rc = self._L.rt_lm_head(self._ctx, _ptr(W_lm), _ptr(g_final), W_lm.shape[0], _ptr(z), int(z_stride), int(B),
                                _ptr(logits))
        _check(self._L, self._ctx, rc)

    # The calls of a serving loop pass addresses as plain integers: a ctypes object per pointer costs as much as the call itself.  What the
    # library cannot see behind an address is checked here: types, entries, inner strides.  The tests on the way of every call are written out
    # in it, a function per tensor takes as long as the tests themselves.
    _known = None

    def _storage(self):
        """What the checks compare with, read from the configuration once."""
        import torch
        cfg = self.cfg
        H, size = cfg.n_heads, 2 if cfg.dtype == RT_BF16 else 4
        self._known = (torch.bfloat16 if size == 2 else torch.float32, torch.int32, torch.float32, cfg.d_model, H, cfg.max_batch,
                       (0, _fit(H, size, cfg.device), _fit(H, 1, cfg.device)), cfg.device)
        return self._known

    def _misfit(self, cache, S):
        fit, lines = cache.fit
        if fit not in self._known[6]:
            _invalid("the cache has %d heads of %d-byte elements on device %d, the context %d of %d or 1 on %d" %
                     (fit >> 16, fit >> 12 & 15, (fit & 4095) - 2, self.cfg.n_heads, 2 if self.cfg.dtype == RT_BF16 else 4, self.cfg.device))
        _invalid("%d sequences and %d lines of the page table" % (S, lines))

    def _rows(self, t, S):
        """Elements between rows that are not simply one behind the other (a dimension of one row has no stride)."""
        shape, stride, d = t.shape, t.stride(), self._known[3]
        if t.dtype is self._known[0] and shape[0] >= S and (
                (len(shape) == 2 and shape[1] == d and stride[1] == 1) or
                (len(shape) == 3 and shape[1] * shape[2] == d and stride[2] == 1 and (stride[1] == shape[2] or shape[1] == 1))):
            return stride[0] if S > 1 else d
        _invalid("rows are [S, n_heads, 64] or [S, d_model] of the storage dtype, contiguous inside")

    def _pairs(self, cache, first, count, k, v):
        dt, i32, _, _, H, _, fits, dev = self._known or self._storage()
        shape, stride, cp = k.shape, k.stride(), None
        if v.stride() == stride and stride[2:] == (64, 1) and v.shape == shape and shape[3] == 64 and shape[2] == H:
            ss, ps, _, _ = stride
        else:
            ss, ps = _pair_strides(k, v, H)
        S = shape[0]
        if k.dtype is not dt or v.dtype is not dt or k.get_device() != dev or v.get_device() != dev or first.get_device() != dev:
            _invalid("k and v are of the storage dtype and, as first and count, on the context's device")
        fit, lines = cache.fit
        if fit not in fits or S > lines:
            self._misfit(cache, S)
        if first.dtype is not i32 or first.numel() < S or not first.is_contiguous():
            _invalid(_INTS)
        if count is not None:
            cp = count.data_ptr()
            if count.dtype is not i32 or count.numel() < S or not count.is_contiguous() or count.get_device() != dev:
                _invalid(_INTS)
        return self._ctx, cache, S, first.data_ptr(), cp, shape[1], k.data_ptr(), v.data_ptr(), ss, ps

    # -- rt_cache_write(ctx, cache, S, first[S] int32, count[S] int32 | None, N, k[S,N,H,64], v, seq_stride, pos_stride)
    def rt_cache_write(self, cache: rt_paged_cache, first, count, k, v):
        rc = self._L.rt_cache_write(*self._pairs(cache, first, count, k, v))
        if rc:
            _check(self._L, self._ctx, rc)

    # -- rt_cache_read(ctx, cache, S, first[S] int32, count[S] int32 | None, N, k[S,N,H,64], v, seq_stride, pos_stride)
    def rt_cache_read(self, cache: rt_paged_cache, first, count, k, v):
        rc = self._L.rt_cache_read(*self._pairs(cache, first, count, k, v))
        if rc:
            _check(self._L, self._ctx, rc)

    # -- rt_paged_attention(ctx, cache, S, lens[S] int32, max_len, q[S,H,64], q_stride, k_t | None, v_t | None, kv_stride, out, out_stride, lse[S,H] f32 | None)
    def rt_paged_attention(self, cache: rt_paged_cache, lens, max_len, q, k_t, v_t, out, lse=None):
        """q, k_t, v_t, out [S, H, 64] (or [S, d]): rows at their first stride, contiguous inside; lse [S, H]."""
        dt, i32, f32, d, H, most, fits, dev = self._known or self._storage()
        S, kp, vp, lp, ks = q.shape[0], None, None, None, d
        fit, lines = cache.fit
        if (fit not in fits or S > lines) and S <= most:   # more than max_batch are refused by the call
            self._misfit(cache, S)
        n = S * d
        qs = d if q.dtype is dt and q.is_contiguous() and q.numel() == n else self._rows(q, S)
        os_ = d if out.dtype is dt and out.is_contiguous() and out.numel() == n else self._rows(out, S)
        if k_t is not None:
            kp, ks = k_t.data_ptr(), d if k_t.dtype is dt and k_t.is_contiguous() and k_t.numel() == n else self._rows(k_t, S)
        if v_t is not None:
            vp, vs = v_t.data_ptr(), d if v_t.dtype is dt and v_t.is_contiguous() and v_t.numel() == n else self._rows(v_t, S)
            if vs != ks and kp is not None:
                _invalid("k_t and v_t have one stride")
        if lse is not None:
            lp = lse.data_ptr()
            if lse.dtype is not f32 or lse.numel() < S * H or not lse.is_contiguous() or lse.get_device() != dev:
                _invalid("lse is contiguous float32 [S, n_heads] on the context's device")
        if lens.dtype is not i32 or lens.numel() < S or not lens.is_contiguous():
            _invalid(_INTS)
        if lens.get_device() != dev or q.get_device() != dev or out.get_device() != dev or (kp and k_t.get_device() != dev) or (vp and v_t.get_device() != dev):
            _invalid("tensors lie on the context's device")
        rc = self._L.rt_paged_attention(self._ctx, cache, S, lens.data_ptr(), max_len, q.data_ptr(), qs, kp, vp, ks, out.data_ptr(), os_, lp)
        if rc:
            _check(self._L, self._ctx, rc)

    # -- rt_decode_step_paged(ctx, w, cache, x_t[S,d], S, pos[S] int32, max_pos, y_t[S,d])
    def rt_decode_step_paged(self, weights: rt_layer_weights, cache: rt_paged_cache, x_t, pos, max_pos, y_t):
        dt, i32, _, d, _, most, fits, dev = self._known or self._storage()
        S = x_t.shape[0]
        fit, lines = cache.fit
        if (fit not in fits or S > lines) and S <= most:   # more than max_batch are refused by the call
            self._misfit(cache, S)
        if x_t.dtype is not dt or y_t.dtype is not dt or not x_t.is_contiguous() or not y_t.is_contiguous() or x_t.numel() != S * d \
                or y_t.numel() < S * d:
            _invalid("x_t and y_t are contiguous [S, d_model] of the storage dtype")
        if pos.dtype is not i32 or pos.numel() < S or not pos.is_contiguous():
            _invalid(_INTS)
        if pos.get_device() != dev or x_t.get_device() != dev or y_t.get_device() != dev:
            _invalid("tensors lie on the context's device")
        rc = self._L.rt_decode_step_paged(self._ctx, weights, cache, x_t.data_ptr(), S, pos.data_ptr(), max_pos, y_t.data_ptr())
        if rc:
            _check(self._L, self._ctx, rc)

    # -- rt_lm_head_mx4(ctx, codes[vocab,d/2], exps[vocab,d/32], g_final[d] | None, vocab, z rows, z_stride, B, logits[B,vocab] f32)
    def rt_lm_head_mx4(self, codes, exps, g_final, z, z_stride, B, logits):
        dt, _, f32, d, _, _, _, dev = self._known or self._storage()
        (vocab, half), gp = codes.shape, None
        if half * 2 != d or exps.numel() != vocab * (d // 32) or codes.element_size() != 1 or exps.element_size() != 1 \
                or not (codes.is_contiguous() and exps.is_contiguous()):
            _invalid("codes [vocab, d / 2] and exps [vocab, d / 32] are contiguous bytes")
        if z.dtype is not dt or not (z.numel() >= (B - 1) * z_stride + d if z.is_contiguous() else
                                     z.shape[0] >= B and z.shape[-1] == d and z.stride(-1) == 1 and (z.stride(0) == z_stride or B == 1)):
            _invalid("z is [B, d] of the storage dtype, its rows contiguous and z_stride apart")
        if logits.dtype is not f32 or logits.numel() < B * vocab or not logits.is_contiguous():
            _invalid("logits are contiguous float32 [B, vocab]")
        if g_final is not None:
            gp = g_final.data_ptr()
            if g_final.dtype is not dt or g_final.numel() != d or not g_final.is_contiguous():
                _invalid("g_final is [d] of the storage dtype")
        if codes.get_device() != dev or exps.get_device() != dev or z.get_device() != dev or logits.get_device() != dev \
                or (gp and g_final.get_device() != dev):
            _invalid("tensors lie on the context's device")
        rc = self._L.rt_lm_head_mx4(self._ctx, codes.data_ptr(), exps.data_ptr(), gp, vocab, z.data_ptr(), z_stride, B, logits.data_ptr())
        if rc:
            _check(self._L, self._ctx, rc)

    # -- rt_cross_block_event(ctx, K, V, B, t1, P, nq)
    def rt_cross_block_event(self, K, V, t1, P, nq):
        rc = self._L.rt_cross_block_event(self._ctx, _ptr(K), _ptr(V), K.shape[1], int(t1), int(P), int(nq))
        _check(self._L, self._ctx, rc)

    def raw_embed(self, table_ptr, vocab, ids_ptr, ids_stride, first, B, N, x_ptr) -> int:
        return self._L.rt_embed_rows(self._ctx, C.c_void_p(table_ptr), vocab, C.c_void_p(ids_ptr), ids_stride, first, B, N,
                                     C.c_void_p(x_ptr))

    def raw_lm_head(self, W_ptr, g_ptr, vocab, z_ptr, z_stride, B, logits_ptr) -> int:
        return self._L.rt_lm_head(self._ctx, C.c_void_p(W_ptr), C.c_void_p(g_ptr), vocab, C.c_void_p(z_ptr), z_stride, B,
                                  C.c_void_p(logits_ptr))

    def raw_prefill(self, weights, x_ptr, B, N, y_ptr, K_ptr, V_ptr, kv_cap) -> int:
        """Status code of rt_layer_prefill on raw addresses (error-path tests)."""
        return self._L.rt_layer_prefill(self._ctx, C.byref(weights) if weights is not None else None, C.c_void_p(x_ptr),
                                        B, N, C.c_void_p(y_ptr), C.c_void_p(K_ptr), C.c_void_p(V_ptr), kv_cap)

    def raw_decode(self, weights, x_ptr, B, t, y_ptr, K_ptr, V_ptr, kv_cap) -> int:
        return self._L.rt_decode_step(self._ctx, C.byref(weights) if weights is not None else None, C.c_void_p(x_ptr),
                                      B, t, C.c_void_p(y_ptr), C.c_void_p(K_ptr), C.c_void_p(V_ptr), kv_cap)

    def last_error(self) -> str:
        return self._L.rt_last_error(self._ctx).decode()

    def engine_name(self) -> str:
        return self._L.rt_engine_name(self._ctx).decode()

    def engine_form(self) -> str:
        return self._L.rt_engine_form(self._ctx).decode()

    def workspace_bytes(self) -> int:
        return int(self._L.rt_workspace_bytes(self._ctx))

    def device_wait_expired(self) -> int:
        return int(self._L.rt_device_wait_expired(self._ctx))

    def phase_trace(self, rows: int):
        """[rows, 16] clock stamps (100 MHz) of the persistent engine, or None when tracing is off."""
        import numpy as np
        buf = np.zeros((rows, 16), dtype=np.uint64)
        n = self._L.rt_phase_trace(self._ctx, buf.ctypes.data_as(C.POINTER(C.c_uint64)), rows)
        return buf[:n] if n > 0 else None

    def decode_phase_trace(self, workgroups: int = 256):
        """[workgroups, 16] clock stamps (100 MHz) of the last single-launch decoding step, or None when tracing is off."""
        import numpy as np
        buf = np.zeros((workgroups, 16), dtype=np.uint64)
        n = self._L.rt_decode_phase_trace(self._ctx, buf.ctypes.data_as(C.POINTER(C.c_uint64)), workgroups)
        return buf[:n] if n > 0 else None

    def rt_destroy(self):
        if self._ctx:
            self._L.rt_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        if _sys is None or _sys.is_finalizing():   # no HIP calls while the interpreter (and the runtimes behind it) shut down
            return
        try:
            self.rt_destroy()
        except Exception:
            pass
