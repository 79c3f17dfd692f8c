"""ctypes binding of libcpattn: the same names as the C entry points, argument marshalling only.

Tensors are ``torch`` CUDA tensors (used for device memory and streams only); every step of the
path runs inside the library's kernels.  The shared library must have been built
(``python -m paper_2609_04774_b200.build``); loading fails loudly otherwise -- there is no
fallback path.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcpattn.so")

CP_OK = 0
CP_ERR_INVALID_ARG, CP_ERR_UNSUPPORTED, CP_ERR_WORKSPACE, CP_ERR_CUDA, CP_ERR_TIMEOUT, CP_ERR_BOUNDS = -1, -2, -3, -4, -5, -6
CP_DTYPE_BF16, CP_DTYPE_F32 = 0, 1
CP_NO_WINDOW = 0x7fffffff

EXPORTS = ["cp_strerror", "cp_last_error", "cp_ctx_create", "cp_ctx_destroy", "cp_ctx_poll_status", "cp_ctx_cache_schedule", "cp_ctx_selftest_wait_expiry", "cp_plan",
           "cp_workspace_bytes", "cp_schedule_inspect", "cp_prefill_attn", "cp_prefill_attn_batch", "cp_prefill_attn_shard", "cp_prefill_attn_chunk", "cp_prefill_attn_kvrange", "cp_prefill_attn_static", "cp_merge",
           "cp_kv_gather", "cp_kv_append", "cp_workspace_bytes_fp8", "cp_prefill_attn_fp8", "cp_prefill_attn_fp8_batch",
           "cp_kv_append_fp8", "cp_kv_append_segments", "cp_prefill_attn_fp8_shard", "cp_prefill_attn_fp8_chunk",
           "cp_prefill_attn_fp8_kvrange", "cp_kv_gather_fp8", "cp_kv_append_segments_fp8", "cp_check_page_table",
           "cp_prefill_attn_window", "cp_prefill_attn_window_batch", "cp_prefill_attn_window_chunk", "cp_prefill_attn_fp8_window_batch",
           "cp_rope_init", "cp_rope_append", "cp_rope_append_fp8", "cp_workspace_bytes_pages", "cp_pages_extend", "cp_pages_evict",
           "cp_pages_free", "cp_pages_fork", "cp_pages_compact", "cp_pages_copy", "cp_workspace_bytes_decode", "cp_decode_attn",
           "cp_decode_attn_fp8"]

# The serving calls run once per layer and token, so their argument types are declared once and plain integers are passed.
_P, _I, _L, _F, _Z = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
_ARGTYPES = {
    "cp_prefill_attn_window": [_P, _P, _P, _P, _L, _L, _I, _L, _L, _I, _F, _P, _P, _P, _Z, _P],
    "cp_prefill_attn_window_batch": [_P, _P, _P, _P, _I, _P, _P, _P, _P, _L, _L, _I, _F, _P, _P, _P, _Z, _P],
    "cp_prefill_attn_window_chunk": [_P, _P, _P, _P, _L, _L, _I, _I, _L, _L, _I, _F, _P, _P, _P, _Z, _P],
    "cp_prefill_attn_fp8_window_batch": [_P, _P, _P, _P, _I, _P, _P, _P, _P, _L, _L, _I, _F, _P, _P, _P, _Z, _P],
    "cp_rope_init": [_P, _I, _P, ctypes.c_double, _I],
    "cp_rope_append": [_P, _P, _P, _P, _P, _L, _I, _P, _P, _P, _P, _P, _L, _L, _P, _P],
    "cp_rope_append_fp8": [_P, _P, _P, _P, _P, _L, _I, _P, _P, _P, _P, _P, _L, _L, _P, _P],
    "cp_workspace_bytes_pages": [_L, _L],
    "cp_pages_extend": [_P, _P, _P, _P, _L, _L, _P, _P, _P, _Z, _P],
    "cp_pages_evict": [_P, _P, _P, _P, _L, _L, _P, _L, _L, _P],
    "cp_pages_free": [_P, _P, _P, _P, _L, _L, _P, _P, _I, _P],
    "cp_pages_fork": [_P, _P, _P, _P, _L, _L, _P, _P, _P, _I, _P, _Z, _P],
    "cp_pages_compact": [_P, _P, _P, _P, _L, _L, _P, _P, _P, _Z, _P],
    "cp_pages_copy": [_P, _P, _P, _P, _I, _P, _Z, _P],
    "cp_workspace_bytes_decode": [_I, _I, _I, _I],
    "cp_decode_attn": [_P, _P, _P, _P, _L, _P, _I, _I, _I, _L, _L, _F, _P, _P, _P, _Z, _P],
    "cp_decode_attn_fp8": [_P, _P, _P, _P, _L, _P, _I, _I, _I, _L, _L, _F, _P, _P, _P, _Z, _P],
}


class CpError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__("%s (%d): %s" % (_strerror(code), code, message))
        self.code = code


class CpArgumentError(CpError, ValueError):
    """A tensor that a call would misread (type, shape, strides, device), refused by the binding."""

    def __init__(self, message: str):
        RuntimeError.__init__(self, "CP_ERR_INVALID_ARG (%d): %s" % (CP_ERR_INVALID_ARG, message))
        self.code = CP_ERR_INVALID_ARG


class cp_shard_plan(ctypes.Structure):
    _fields_ = [("q_begin", ctypes.c_int64 * 2), ("q_end", ctypes.c_int64 * 2), ("kv_end", ctypes.c_int64 * 2),
                ("pairs", ctypes.c_uint64)]


class cp_kv_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("num_pages", ctypes.c_int64),
                ("page_size", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("stride_page", ctypes.c_int64), ("stride_tok", ctypes.c_int64),
                ("stride_head", ctypes.c_int64)]


class cp_kv_cache_fp8(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("num_pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("stride_page", ctypes.c_int64), ("stride_tok", ctypes.c_int64),
                ("stride_head", ctypes.c_int64)]


class cp_rope(ctypes.Structure):
    _fields_ = [("n_axes", ctypes.c_int32), ("rot_dims", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("axis", ctypes.c_int32 * 64), ("freq", ctypes.c_double * 64)]


class cp_page_pool(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("num_pages", ctypes.c_int64), ("n_layers", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("row_bytes", ctypes.c_int32), ("stride_page", ctypes.c_int64),
                ("stride_tok", ctypes.c_int64), ("stride_head", ctypes.c_int64)]


_lib = None


def load():
    """Load libcpattn.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libcpattn.so is missing at %s: run `python -m paper_2609_04774_b200.build` "
                               "(there is no fallback implementation)" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        lib.cp_strerror.restype = ctypes.c_char_p
        lib.cp_strerror.argtypes = [ctypes.c_int]
        lib.cp_last_error.restype = ctypes.c_char_p
        lib.cp_workspace_bytes.restype = ctypes.c_size_t
        lib.cp_workspace_bytes_fp8.restype = ctypes.c_size_t
        lib.cp_workspace_bytes_pages.restype = ctypes.c_size_t
        lib.cp_workspace_bytes_decode.restype = ctypes.c_size_t
        for name in EXPORTS:
            if name not in ("cp_strerror", "cp_last_error") and not name.startswith("cp_workspace_bytes"):
                getattr(lib, name).restype = ctypes.c_int
        for name, types in _ARGTYPES.items():
            getattr(lib, name).argtypes = types
        _lib = lib
    return _lib


def _strerror(code: int) -> str:
    return load().cp_strerror(code).decode()


def _check(rc: int) -> None:
    if rc != CP_OK:
        raise CpError(rc, load().cp_last_error().decode())


def _ptr(t):
    return ctypes.c_void_p(0 if t is None else t.data_ptr())


def _i64(a):
    return np.ascontiguousarray(a, dtype=np.int64)


def _i32(a):
    return np.ascontiguousarray(a, dtype=np.int32)


def _hp(a):
    """Address of a host numpy array (the plain integer route; `ctypes.data_as` costs twice as much per call)."""
    return ctypes.c_void_p(a.ctypes.data)


def _stream(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


class Context:
    """cp_ctx handle (cp_ctx_create / cp_ctx_destroy / cp_ctx_poll_status)."""

    def __init__(self, device: int = 0):
        self._h = ctypes.c_void_p()
        _check(load().cp_ctx_create(ctypes.byref(self._h), ctypes.c_int(device)))
        self.device = device

    def close(self):
        if self._h:
            load().cp_ctx_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def cache_schedule(self, enable: bool):
        """Reuse the work lists left in the workspace by the previous call when the next one has the same shape."""
        _check(load().cp_ctx_cache_schedule(self._h, ctypes.c_int(1 if enable else 0)))

    def selftest_wait_expiry(self, stream=None):
        """Enqueue the bounded-wait self-test; the next poll_status() after a sync raises CP_ERR_TIMEOUT."""
        _check(load().cp_ctx_selftest_wait_expiry(self._h, _stream(stream)))

    def poll_status(self):
        """Raises CpError if a device-side wait expired since the last poll."""
        detail = (ctypes.c_int32 * 4)()
        _check(load().cp_ctx_poll_status(self._h, detail))


def cp_plan(new_len: int, prefix_len: int, C: int):
    """Zigzag shard plan: list of C dicts {q_begin, q_end, kv_end, pairs}."""
    arr = (cp_shard_plan * max(C, 1))()
    _check(load().cp_plan(ctypes.c_int64(new_len), ctypes.c_int64(prefix_len), ctypes.c_int32(C), arr))
    return [{"q_begin": list(s.q_begin), "q_end": list(s.q_end), "kv_end": list(s.kv_end), "pairs": int(s.pairs)}
            for s in arr[:C]]


def cp_workspace_bytes(new_len, C, Hq) -> int:
    nl, cs = _i64(new_len).reshape(-1), _i32(C).reshape(-1)
    return int(load().cp_workspace_bytes(ctypes.c_int32(nl.size), _hp(nl),
                                         _hp(cs), ctypes.c_int32(Hq)))


def cp_schedule_inspect(cu_new, prefix_len, C, Hq, Hkv, num_sms=148, want_lists=True):
    """Host-only view of the varlen tile schedule: (summary dict, pieces [n,6] int32, items [n,4] int32)."""
    cu_new, prefix_len, C = _i64(cu_new), _i64(prefix_len), _i32(C)
    B = prefix_len.size
    summary = np.zeros(10, dtype=np.int64)
    args = [ctypes.c_int32(B), _hp(cu_new), _hp(prefix_len),
            _hp(C), ctypes.c_int32(Hq), ctypes.c_int32(Hkv), ctypes.c_int32(num_sms),
            _hp(summary)]
    _check(load().cp_schedule_inspect(*args, None, ctypes.c_int64(0), None, ctypes.c_int64(0)))
    keys = ["grid", "tiles", "pieces", "split_units", "slots", "max_load", "min_load", "total", "inline", "launches"]
    info = dict(zip(keys, (int(x) for x in summary)))
    if not want_lists:
        return info, None, None
    pieces = np.zeros((info["pieces"], 6), dtype=np.int32)
    items = np.zeros((info["tiles"], 4), dtype=np.int32)
    _check(load().cp_schedule_inspect(*args, _hp(pieces), ctypes.c_int64(pieces.shape[0]),
                                      _hp(items), ctypes.c_int64(items.shape[0])))
    return info, pieces, items


def _paged(pools, dtypes, what):
    """Device of paged tensors [num_pages, page_size, Hkv, D] of one shape, type and layout on one device, refused otherwise: the kernels
    compute every address from the first one's."""
    first = pools[0]
    if first.dim() != 4 or first.stride(3) != 1:
        raise CpArgumentError("%s: K and V are [num_pages, page_size, Hkv, D] with unit stride in the last dimension, got %s with strides %s"
                              % (what, tuple(first.shape), first.stride()))
    for t in pools[1:]:
        if t.shape != first.shape or t.stride() != first.stride() or t.dtype != first.dtype or t.device != first.device:
            raise CpArgumentError("%s: K and V must agree in shape, strides, type and device, got %s %s with strides %s on %s and %s %s with strides "
                                  "%s on %s" % (what, first.dtype, tuple(first.shape), first.stride(), first.device, t.dtype, tuple(t.shape),
                                                t.stride(), t.device))
    if str(first.dtype) not in dtypes:
        raise CpArgumentError("%s: K and V are %s, got %s" % (what, " or ".join(dtypes), first.dtype))
    if not first.is_cuda:
        raise CpArgumentError("%s: K and V must be on a CUDA device, got %s" % (what, first.device))
    return first.get_device()


_BF16, _CODES = ("torch.bfloat16",), ("torch.uint8", "torch.int8", "torch.float8_e4m3fn")


def make_cache(k_pages, v_pages) -> cp_kv_cache:
    """Describe paged K/V tensors [num_pages, page_size, Hkv, D] (bf16, any strides with dim stride 1)."""
    device = _paged((k_pages, v_pages), _BF16, "make_cache")
    c = cp_kv_cache()
    c.device = device                                      # compared with the context's by the serving calls
    c.k, c.v = k_pages.data_ptr(), v_pages.data_ptr()
    c.num_pages, c.page_size, c.Hkv, c.D = k_pages.shape
    c.stride_page, c.stride_tok, c.stride_head = k_pages.stride(0), k_pages.stride(1), k_pages.stride(2)
    return c


def cp_prefill_attn(ctx, q, cache, page_table, prefix_len, new_len, C, Hq, scale, out, lse, workspace, stream=None):
    _check(load().cp_prefill_attn(ctx._h, _ptr(q), ctypes.byref(cache), _ptr(page_table), ctypes.c_int64(prefix_len),
                                  ctypes.c_int64(new_len), ctypes.c_int32(C), ctypes.c_int32(Hq),
                                  ctypes.c_float(scale), _ptr(out), _ptr(lse), _ptr(workspace),
                                  ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream(stream)))


def cp_prefill_attn_batch(ctx, q, cache, page_table, cu_new, prefix_len, C, cu_pages, Hq, scale, out, lse, workspace,
                          stream=None):
    cu_new, prefix_len, cu_pages, C = _i64(cu_new), _i64(prefix_len), _i64(cu_pages), _i32(C)
    B = prefix_len.size
    assert cu_new.size == B + 1 and cu_pages.size == B + 1 and C.size == B
    _check(load().cp_prefill_attn_batch(
        ctx._h, _ptr(q), ctypes.byref(cache), _ptr(page_table), ctypes.c_int32(B),
        _hp(cu_new), _hp(prefix_len),
        _hp(C), _hp(cu_pages), ctypes.c_int32(Hq),
        ctypes.c_float(scale), _ptr(out), _ptr(lse), _ptr(workspace),
        ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream(stream)))


def cp_prefill_attn_shard(ctx, q, cache, page_table, prefix_len, new_len, C, shard, Hq, scale, partial_out,
                          partial_lse, workspace, stream=None):
    _check(load().cp_prefill_attn_shard(
        ctx._h, _ptr(q), ctypes.byref(cache), _ptr(page_table), ctypes.c_int64(prefix_len), ctypes.c_int64(new_len),
        ctypes.c_int32(C), ctypes.c_int32(shard), ctypes.c_int32(Hq), ctypes.c_float(scale), _ptr(partial_out),
        _ptr(partial_lse), _ptr(workspace), ctypes.c_size_t(workspace.numel() * workspace.element_size()),
        _stream(stream)))


def cp_prefill_attn_chunk(ctx, q_chunk, cache, page_table, prefix_len, new_len, C, chunk, Hq, scale, out_chunk,
                          lse_chunk, workspace, stream=None):
    """One zigzag chunk in chunk-local buffers: q_chunk/out_chunk [n,Hq,D] bf16, lse_chunk [Hq,n] fp32."""
    _check(load().cp_prefill_attn_chunk(
        ctx._h, _ptr(q_chunk), ctypes.byref(cache), _ptr(page_table), ctypes.c_int64(prefix_len),
        ctypes.c_int64(new_len), ctypes.c_int32(C), ctypes.c_int32(chunk), ctypes.c_int32(Hq), ctypes.c_float(scale),
        _ptr(out_chunk), _ptr(lse_chunk), _ptr(workspace),
        ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream(stream)))


def cp_prefill_attn_kvrange(ctx, q, cache, page_table, prefix_len, new_len, kv_lo, kv_hi, Hq, scale, partial_out,
                            partial_lse, workspace, stream=None):
    """All R queries against keys at absolute positions [kv_lo, kv_hi) only: fp32 partial + LSE for cp_merge."""
    _check(load().cp_prefill_attn_kvrange(
        ctx._h, _ptr(q), ctypes.byref(cache), _ptr(page_table), ctypes.c_int64(prefix_len), ctypes.c_int64(new_len),
        ctypes.c_int64(kv_lo), ctypes.c_int64(kv_hi), ctypes.c_int32(Hq), ctypes.c_float(scale), _ptr(partial_out),
        _ptr(partial_lse), _ptr(workspace), ctypes.c_size_t(workspace.numel() * workspace.element_size()),
        _stream(stream)))


def _window_args(kind, ctx, q, cache, page_table, rows, Hq, out, lse, workspace, stream):
    """The tensors of a windowed call, checked: (q, cache, page_table) and (out, lse, workspace, its bytes, stream)."""
    bf16, i32, f32, _ = _types or _torch_types()
    shape = (rows, Hq, 128)
    table = _arg(ctx, page_table, "page_table", i32, page_table.shape)
    ws, ws_bytes = _workspace(ctx, workspace)
    qp, op, lp = _arg(ctx, q, "q", bf16, shape), _arg(ctx, out, "out", bf16, shape), _arg(ctx, lse, "lse", f32, (Hq, rows))
    if rows == 0:                                          # an empty chunk: empty tensors have no address, the call reads none
        qp = op = lp = ws
    return (ctx._h, qp, _described(ctx, cache, kind), table), (op, lp, ws, ws_bytes, _raw_stream(ctx, stream))


def _host_i64(a):
    """ctypes array of 64-bit integers from a list, tuple or array."""
    return (ctypes.c_int64 * len(a))(*a)


def cp_prefill_attn_window(ctx, q, cache, page_table, prefix_len, new_len, C, window, sinks, Hq, scale, out, lse, workspace,
                           stream=None):
    """cp_prefill_attn where a token at position p sees the last `window` keys (its own among them) and the first `sinks`."""
    head, tail = _window_args(cp_kv_cache, ctx, q, cache, page_table, new_len, Hq, out, lse, workspace, stream)
    if page_table.numel() * cache.page_size < prefix_len + new_len:
        raise CpArgumentError("page_table has %d entries for %d tokens" % (page_table.numel(), prefix_len + new_len))
    _check(load().cp_prefill_attn_window(*head, prefix_len, new_len, C, window, sinks, Hq, scale, *tail))


def _window_batch(call, kind, ctx, q, cache, page_table, cu_new, prefix_len, C, cu_pages, window, sinks, Hq, scale, out, lse,
                  workspace, stream):
    B = len(prefix_len)
    if len(cu_new) != B + 1 or len(cu_pages) != B + 1 or len(C) != B:
        raise CpArgumentError("cu_new and cu_pages have %d and %d entries, C %d, for %d requests" % (len(cu_new), len(cu_pages), len(C), B))
    head, tail = _window_args(kind, ctx, q, cache, page_table, int(cu_new[B]), Hq, out, lse, workspace, stream)
    if page_table.numel() < cu_pages[B]:
        raise CpArgumentError("page_table has %d entries, cu_pages ends with %d" % (page_table.numel(), cu_pages[B]))
    _check(call(*head, B, _host_i64(cu_new), _host_i64(prefix_len), (ctypes.c_int32 * B)(*C), _host_i64(cu_pages), window, sinks, Hq, scale, *tail))


def cp_prefill_attn_window_batch(ctx, q, cache, page_table, cu_new, prefix_len, C, cu_pages, window, sinks, Hq, scale, out, lse,
                                 workspace, stream=None):
    """B requests in one launch; cu_new, prefix_len, C, cu_pages: host sequences as in cp_prefill_attn_batch."""
    _window_batch(load().cp_prefill_attn_window_batch, cp_kv_cache, ctx, q, cache, page_table, cu_new, prefix_len, C, cu_pages,
                  window, sinks, Hq, scale, out, lse, workspace, stream)


def cp_prefill_attn_window_chunk(ctx, q_chunk, cache, page_table, prefix_len, new_len, C, chunk, window, sinks, Hq, scale,
                                 out_chunk, lse_chunk, workspace, stream=None):
    """One zigzag chunk in chunk-local buffers, as cp_prefill_attn_chunk, with a window."""
    if C >= 1 and 0 <= chunk < 2 * C and new_len >= 1 and prefix_len >= 0:
        cl = -(-new_len // (2 * C))
        rows, end = min(new_len, (chunk + 1) * cl) - min(new_len, chunk * cl), prefix_len + min(new_len, (chunk + 1) * cl)
        if page_table.numel() * cache.page_size < end:
            raise CpArgumentError("page_table has %d entries for %d tokens" % (page_table.numel(), end))
    else:
        rows = q_chunk.shape[0]                            # refused by the call
    head, tail = _window_args(cp_kv_cache, ctx, q_chunk, cache, page_table, rows, Hq, out_chunk, lse_chunk, workspace, stream)
    _check(load().cp_prefill_attn_window_chunk(*head, prefix_len, new_len, C, chunk, window, sinks, Hq, scale, *tail))


def cp_prefill_attn_static(q, cache, page_table, prefix_len, new_len, C, Hq, scale, out, lse, stream=None):
    """cp_prefill_attn without a context or a workspace: the library's built-in device scratch holds the
    tile list, so nothing is allocated.  For callers that cannot allocate device memory (all of HBM
    already handed to a cache pool, allocation-free serving loops).  Limits: ceil(new_len/128) + 2*C <= 2048
    tiles; calls share the scratch, so calls that may overlap on the GPU must be ordered by the caller."""
    _check(load().cp_prefill_attn_static(_ptr(q), ctypes.byref(cache), _ptr(page_table), ctypes.c_int64(prefix_len),
                                         ctypes.c_int64(new_len), ctypes.c_int32(C), ctypes.c_int32(Hq),
                                         ctypes.c_float(scale), _ptr(out), _ptr(lse), _stream(stream)))


def cp_merge(ctx, partials, lses, out, lse_out=None, stream=None):
    """partials [N,T,H,D] fp32, lses [N,H,T] fp32 -> out [T,H,D] (bf16 or fp32), lse_out [H,T] or None."""
    import torch
    N, T, H, D = partials.shape
    dt = CP_DTYPE_BF16 if out.dtype == torch.bfloat16 else CP_DTYPE_F32
    _check(load().cp_merge(ctx._h, _ptr(partials), _ptr(lses), ctypes.c_int32(N), ctypes.c_int64(T),
                           ctypes.c_int32(H), ctypes.c_int32(D), _ptr(out), ctypes.c_int32(dt), _ptr(lse_out),
                           _stream(stream)))


def cp_kv_gather(ctx, cache, page_table, t_begin, n, k_rows, v_rows, stream=None):
    _check(load().cp_kv_gather(ctx._h, ctypes.byref(cache), _ptr(page_table), ctypes.c_int64(t_begin),
                               ctypes.c_int64(n), _ptr(k_rows), _ptr(v_rows), _stream(stream)))


def cp_kv_append(ctx, cache, page_table, t_begin, n, k_rows, v_rows, stream=None):
    _check(load().cp_kv_append(ctx._h, ctypes.byref(cache), _ptr(page_table), ctypes.c_int64(t_begin),
                               ctypes.c_int64(n), _ptr(k_rows), _ptr(v_rows), _stream(stream)))


def cp_kv_append_segments(ctx, cache, page_table, segments, k_rows, v_rows, stream=None):
    """segments: iterable of (t_begin, n, row0); rows [row0, row0+n) of k_rows / v_rows go to tokens [t_begin, t_begin+n)."""
    seg = np.ascontiguousarray(np.asarray(list(segments), dtype=np.int64).reshape(-1, 3))
    _check(load().cp_kv_append_segments(ctx._h, ctypes.byref(cache), _ptr(page_table), ctypes.c_int32(seg.shape[0]),
                                        _hp(seg), _ptr(k_rows), _ptr(v_rows), _stream(stream)))


# ------------------------------------------------------------------------------------------------
# FP8 K/V variant
# ------------------------------------------------------------------------------------------------

def make_cache_fp8(k8_pages, v8_pages, k_scale, v_scale) -> cp_kv_cache_fp8:
    """Describe paged E4M3 K/V tensors [num_pages, page_size, Hkv, D] (uint8) with fp32 scales [Hkv] on the device."""
    scales = (("k_scale", k_scale), ("v_scale", v_scale))
    for name, t in scales:
        if k8_pages.dim() == 4 and (str(t.dtype) != "torch.float32" or t.numel() != k8_pages.shape[2] or not t.is_contiguous()):
            raise CpArgumentError("make_cache_fp8: %s must be a contiguous fp32 tensor of %d elements (one per KV head), got %s %s with strides %s"
                                  % (name, k8_pages.shape[2], t.dtype, tuple(t.shape), t.stride()))
    device = _paged((k8_pages, v8_pages), _CODES, "make_cache_fp8")
    for name, t in scales:
        if t.device != k8_pages.device:
            raise CpArgumentError("make_cache_fp8: %s is on %s, the pages are on %s" % (name, t.device, k8_pages.device))
    c = cp_kv_cache_fp8()
    c.device = device
    c.k, c.v, c.k_scale, c.v_scale = k8_pages.data_ptr(), v8_pages.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr()
    c.num_pages, c.page_size, c.Hkv, c.D = k8_pages.shape
    c.stride_page, c.stride_tok, c.stride_head = k8_pages.stride(0), k8_pages.stride(1), k8_pages.stride(2)
    return c


def cp_workspace_bytes_fp8(new_len, C, Hq) -> int:
    nl, cs = _i64(new_len).reshape(-1), _i32(C).reshape(-1)
    return int(load().cp_workspace_bytes_fp8(ctypes.c_int32(nl.size), _hp(nl), _hp(cs), ctypes.c_int32(Hq)))


def cp_prefill_attn_fp8(ctx, q, cache, page_table, prefix_len, new_len, C, Hq, scale, out, lse, workspace, stream=None):
    _check(load().cp_prefill_attn_fp8(ctx._h, _ptr(q), ctypes.byref(cache), _ptr(page_table), ctypes.c_int64(prefix_len),
                                      ctypes.c_int64(new_len), ctypes.c_int32(C), ctypes.c_int32(Hq),
                                      ctypes.c_float(scale), _ptr(out), _ptr(lse), _ptr(workspace),
                                      ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream(stream)))


def cp_prefill_attn_fp8_batch(ctx, q, cache, page_table, cu_new, prefix_len, C, cu_pages, Hq, scale, out, lse, workspace,
                              stream=None):
    cu_new, prefix_len, cu_pages, C = _i64(cu_new), _i64(prefix_len), _i64(cu_pages), _i32(C)
    B = prefix_len.size
    assert cu_new.size == B + 1 and cu_pages.size == B + 1 and C.size == B
    _check(load().cp_prefill_attn_fp8_batch(
        ctx._h, _ptr(q), ctypes.byref(cache), _ptr(page_table), ctypes.c_int32(B), _hp(cu_new), _hp(prefix_len), _hp(C),
        _hp(cu_pages), ctypes.c_int32(Hq), ctypes.c_float(scale), _ptr(out), _ptr(lse), _ptr(workspace),
        ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream(stream)))


def cp_prefill_attn_fp8_window_batch(ctx, q, cache, page_table, cu_new, prefix_len, C, cu_pages, window, sinks, Hq, scale, out,
                                     lse, workspace, stream=None):
    _window_batch(load().cp_prefill_attn_fp8_window_batch, cp_kv_cache_fp8, ctx, q, cache, page_table, cu_new, prefix_len, C, cu_pages,
                  window, sinks, Hq, scale, out, lse, workspace, stream)


def cp_prefill_attn_fp8_shard(ctx, q, cache, page_table, prefix_len, new_len, C, shard, Hq, scale, partial_out, partial_lse,
                              workspace, stream=None):
    _check(load().cp_prefill_attn_fp8_shard(
        ctx._h, _ptr(q), ctypes.byref(cache), _ptr(page_table), ctypes.c_int64(prefix_len), ctypes.c_int64(new_len),
        ctypes.c_int32(C), ctypes.c_int32(shard), ctypes.c_int32(Hq), ctypes.c_float(scale), _ptr(partial_out),
        _ptr(partial_lse), _ptr(workspace), ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream(stream)))


def cp_prefill_attn_fp8_chunk(ctx, q_chunk, cache, page_table, prefix_len, new_len, C, chunk, Hq, scale, out_chunk, lse_chunk,
                              workspace, stream=None):
    _check(load().cp_prefill_attn_fp8_chunk(
        ctx._h, _ptr(q_chunk), ctypes.byref(cache), _ptr(page_table), ctypes.c_int64(prefix_len), ctypes.c_int64(new_len),
        ctypes.c_int32(C), ctypes.c_int32(chunk), ctypes.c_int32(Hq), ctypes.c_float(scale), _ptr(out_chunk), _ptr(lse_chunk),
        _ptr(workspace), ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream(stream)))


def cp_prefill_attn_fp8_kvrange(ctx, q, cache, page_table, prefix_len, new_len, kv_lo, kv_hi, Hq, scale, partial_out,
                                partial_lse, workspace, stream=None):
    _check(load().cp_prefill_attn_fp8_kvrange(
        ctx._h, _ptr(q), ctypes.byref(cache), _ptr(page_table), ctypes.c_int64(prefix_len), ctypes.c_int64(new_len),
        ctypes.c_int64(kv_lo), ctypes.c_int64(kv_hi), ctypes.c_int32(Hq), ctypes.c_float(scale), _ptr(partial_out),
        _ptr(partial_lse), _ptr(workspace), ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream(stream)))


def cp_kv_append_fp8(ctx, cache, page_table, t_begin, n, k_rows, v_rows, stream=None):
    """bf16 rows [n, Hkv, D] -> E4M3 bytes of logical tokens t_begin.. of the FP8 cache (per-head scales)."""
    _check(load().cp_kv_append_fp8(ctx._h, ctypes.byref(cache), _ptr(page_table), ctypes.c_int64(t_begin),
                                   ctypes.c_int64(n), _ptr(k_rows), _ptr(v_rows), _stream(stream)))


def cp_kv_gather_fp8(ctx, cache, page_table, t_begin, n, k_bytes, v_bytes, stream=None):
    """Raw E4M3 bytes of logical tokens [t_begin, t_begin + n) -> k_bytes / v_bytes [n, Hkv, D] uint8."""
    _check(load().cp_kv_gather_fp8(ctx._h, ctypes.byref(cache), _ptr(page_table), ctypes.c_int64(t_begin),
                                   ctypes.c_int64(n), _ptr(k_bytes), _ptr(v_bytes), _stream(stream)))


def cp_kv_append_segments_fp8(ctx, cache, page_table, segments, k_bytes, v_bytes, stream=None):
    """cp_kv_append_segments for an FP8 cache: rows of stored bytes, copied as they are."""
    seg = np.ascontiguousarray(np.asarray(list(segments), dtype=np.int64).reshape(-1, 3))
    _check(load().cp_kv_append_segments_fp8(ctx._h, ctypes.byref(cache), _ptr(page_table), ctypes.c_int32(seg.shape[0]),
                                            _hp(seg), _ptr(k_bytes), _ptr(v_bytes), _stream(stream)))


def cp_check_page_table(ctx, page_table, num_pages, stream=None):
    """Enqueue the page-table check; a bad entry shows as CP_ERR_BOUNDS at the next poll_status() after a sync."""
    _check(load().cp_check_page_table(ctx._h, _ptr(page_table), ctypes.c_int64(page_table.numel()),
                                      ctypes.c_int64(num_pages), _stream(stream)))


# ------------------------------------------------------------------------------------------------
# Serving calls: decode attention, rotary append, page care
# ------------------------------------------------------------------------------------------------

_types = None      # (bf16, int32, float32, the current raw stream of a device), from torch at the first call


def _torch_types():
    global _types
    import torch
    _types = (torch.bfloat16, torch.int32, torch.float32, torch._C._cuda_getCurrentRawStream)
    return _types


def _raw_stream(ctx, stream):
    """The given stream, or the current one of the context's device."""
    return stream.cuda_stream if stream is not None else _types[3](ctx.device)


def _arg(ctx, t, name, dtype, shape):
    """Address of a contiguous tensor of the given type and shape on the context's device."""
    if t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == ctx.device:
        return t.data_ptr()
    raise CpArgumentError("%s must be a contiguous %s tensor of shape %s on cuda:%d, got %s %s with strides %s on %s"
                     % (name, dtype, tuple(shape), ctx.device, t.dtype, tuple(t.shape), t.stride(), t.device))


def _described(ctx, desc, kind):
    """Address of a descriptor, which must be of the kind that the call reads and, unless made by hand, of tensors on the context's device."""
    if not isinstance(desc, kind):
        raise CpArgumentError("the call takes a %s, got a %s" % (kind.__name__, type(desc).__name__))
    if getattr(desc, "device", ctx.device) != ctx.device:
        raise CpArgumentError("the %s describes tensors on cuda:%d, the context is on cuda:%d" % (kind.__name__, desc.device, ctx.device))
    return ctypes.addressof(desc)


def _workspace(ctx, t):
    if not t.is_contiguous() or t.get_device() != ctx.device:
        raise CpArgumentError("workspace must be a contiguous tensor on cuda:%d" % ctx.device)
    return t.data_ptr(), t.nbytes


def cp_workspace_bytes_decode(B, n_q, Hq, Hkv) -> int:
    return int(load().cp_workspace_bytes_decode(B, n_q, Hq, Hkv))


def _decode_attn(call, kind, ctx, q, cache, page_table, kv_len, window, sinks, scale, out, lse, workspace, stream):
    bf16, i32, f32, _ = _types or _torch_types()
    shape = q.shape
    B, n_q, Hq, _ = shape
    stride = page_table.shape[1]
    ws, ws_bytes = _workspace(ctx, workspace)
    rc = call(ctx._h, _arg(ctx, q, "q", bf16, (B, n_q, Hq, 128)), _described(ctx, cache, kind), _arg(ctx, page_table, "page_table", i32, (B, stride)), stride,
              _arg(ctx, kv_len, "kv_len", i32, (B,)), B, n_q, Hq, window, sinks, scale, _arg(ctx, out, "out", bf16, shape),
              _arg(ctx, lse, "lse", f32, (Hq, B * n_q)), ws, ws_bytes, _raw_stream(ctx, stream))
    if rc != CP_OK:
        _check(rc)


def cp_decode_attn(ctx, q, cache, page_table, kv_len, window, sinks, scale, out, lse, workspace, stream=None):
    """The last n_q tokens of B sequences: q, out [B, n_q, Hq, 128] bf16, page_table [B, stride] and kv_len [B] int32 on the device (new
    tokens included), lse [Hq, B * n_q] fp32.  window = CP_NO_WINDOW: every key."""
    _decode_attn(load().cp_decode_attn, cp_kv_cache, ctx, q, cache, page_table, kv_len, window, sinks, scale, out, lse, workspace, stream)


def cp_decode_attn_fp8(ctx, q, cache, page_table, kv_len, window, sinks, scale, out, lse, workspace, stream=None):
    """cp_decode_attn over an FP8 cache."""
    _decode_attn(load().cp_decode_attn_fp8, cp_kv_cache_fp8, ctx, q, cache, page_table, kv_len, window, sinks, scale, out, lse, workspace, stream)


def make_rope(sections, base=10000.0, interleaved=False) -> cp_rope:
    """Rotary description for consecutive sections of pairs, one per axis ([64]: plain positions; [16, 24, 24]: time, height, width).
    Its axis[] and freq[] (radians per position, per pair) may be changed afterwards."""
    sec = _i32(sections).reshape(-1)
    rope = cp_rope()
    _check(load().cp_rope_init(ctypes.addressof(rope), sec.size, sec.ctypes.data, base, 1 if interleaved else 0))
    return rope


def _rope_append(call, kind, ctx, rope, q, k_rows, v_rows, positions, token_seq, token_slot, cache, page_table, q_out, stream):
    bf16, i32, _, _ = _types or _torch_types()
    n = token_seq.shape[0]
    qp = qo = kp = vp = sp = tp = None
    Hq = rows = stride = 0
    if q is not None or q_out is not None:
        if q is None or q_out is None:
            raise CpArgumentError("q and q_out come together or not at all")
        Hq = q.shape[1]
        qp, qo = _arg(ctx, q, "q", bf16, (n, Hq, 128)), _arg(ctx, q_out, "q_out", bf16, (n, Hq, 128))
    if k_rows is not None or v_rows is not None:
        if k_rows is None or v_rows is None:
            raise CpArgumentError("k_rows and v_rows come together or not at all")
        shape = (n, cache.Hkv, 128)
        rows, stride = page_table.shape
        kp, vp = _arg(ctx, k_rows, "k_rows", bf16, shape), _arg(ctx, v_rows, "v_rows", bf16, shape)
        sp, tp = _arg(ctx, token_slot, "token_slot", i32, (n,)), _arg(ctx, page_table, "page_table", i32, (rows, stride))
    rc = call(ctx._h, _described(ctx, rope, cp_rope), qp, kp, vp, n, Hq, _arg(ctx, positions, "positions", i32, (rope.n_axes, n)),
              _arg(ctx, token_seq, "token_seq", i32, (n,)), sp, _described(ctx, cache, kind), tp, rows, stride, qo, _raw_stream(ctx, stream))
    if rc != CP_OK:
        _check(rc)


def cp_rope_append(ctx, rope, q, k_rows, v_rows, positions, token_seq, token_slot, cache, page_table, q_out, stream=None):
    """q [n, Hq, 128] -> q_out (may be q); k_rows, v_rows [n, Hkv, 128] -> slot token_slot[i] of sequence token_seq[i] of the paged cache;
    positions [n_axes, n], token_seq, token_slot [n], page_table [rows, stride], all int32.  token_seq < 0: padding."""
    _rope_append(load().cp_rope_append, cp_kv_cache, ctx, rope, q, k_rows, v_rows, positions, token_seq, token_slot, cache, page_table, q_out, stream)


def cp_rope_append_fp8(ctx, rope, q, k_rows, v_rows, positions, token_seq, token_slot, cache, page_table, q_out, stream=None):
    """cp_rope_append into an FP8 cache: k (rotated) and v as e4m3(x / scale[head])."""
    _rope_append(load().cp_rope_append_fp8, cp_kv_cache_fp8, ctx, rope, q, k_rows, v_rows, positions, token_seq, token_slot, cache, page_table, q_out, stream)


def make_page_pool(k, v, num_pages=None) -> cp_page_pool:
    """Describe the K and V pools of one numbering of pages: k, v [layers, num_pages, page_size, Hkv, 128], or lists of such 4-D
    tensors, bf16 or uint8 (E4M3); all of one geometry."""
    ks, vs = [k[i] for i in range(len(k))], [v[i] for i in range(len(v))]
    if len(ks) != len(vs) or not ks:
        raise CpArgumentError("make_page_pool: %d layers of k, %d of v" % (len(ks), len(vs)))
    device = _paged(ks + vs, _BF16 + _CODES, "make_page_pool")
    first = ks[0]
    if first.shape[3] != 128 or (num_pages is not None and num_pages != first.shape[0]):
        raise CpArgumentError("a layer is [num_pages, page_size, Hkv, 128], got %s" % (tuple(first.shape),))
    e = first.element_size()
    p = cp_page_pool()
    p.device = device
    p._k = (ctypes.c_void_p * len(ks))(*[t.data_ptr() for t in ks])        # kept alive with the descriptor
    p._v = (ctypes.c_void_p * len(vs))(*[t.data_ptr() for t in vs])
    p.k, p.v = ctypes.addressof(p._k), ctypes.addressof(p._v)
    p.n_layers = len(ks)
    p.num_pages, p.page_size, p.Hkv, p.row_bytes = first.shape[0], first.shape[1], first.shape[2], 128 * e
    p.stride_page, p.stride_tok, p.stride_head = first.stride(0) * e, first.stride(1) * e, first.stride(2) * e
    return p


def cp_workspace_bytes_pages(num_pages, n=0) -> int:
    return int(load().cp_workspace_bytes_pages(num_pages, n))


def _table_args(ctx, pool, refcount, page_table):
    i32 = (_types or _torch_types())[1]
    rows, stride = page_table.shape
    return (ctx._h, _described(ctx, pool, cp_page_pool), _arg(ctx, refcount, "refcount", i32, (pool.num_pages,)),
            _arg(ctx, page_table, "page_table", i32, (rows, stride)), rows, stride)


def _ints(ctx, t, name, n):
    return _arg(ctx, t, name, _types[1], (n,))


def cp_pages_extend(ctx, pool, refcount, page_table, kv_len, new_tokens, workspace, stream=None):
    """Room for new_tokens[r] more tokens in every row: entries, references and kv_len are updated on the device."""
    a = _table_args(ctx, pool, refcount, page_table)
    _check(load().cp_pages_extend(*a, _ints(ctx, kv_len, "kv_len", a[4]), _ints(ctx, new_tokens, "new_tokens", a[4]), *_workspace(ctx, workspace),
                                  _raw_stream(ctx, stream)))


def cp_pages_evict(ctx, pool, refcount, page_table, kv_len, window, sinks, stream=None):
    """Give back the pages that the next token of each row (position kv_len) and all later ones cannot see."""
    a = _table_args(ctx, pool, refcount, page_table)
    _check(load().cp_pages_evict(*a, _ints(ctx, kv_len, "kv_len", a[4]), window, sinks, _raw_stream(ctx, stream)))


def cp_pages_free(ctx, pool, refcount, page_table, kv_len, rows, stream=None):
    """Give back all pages of the listed rows (int32 tensor); their kv_len becomes 0."""
    a = _table_args(ctx, pool, refcount, page_table)
    n = rows.numel()
    _check(load().cp_pages_free(*a, _ints(ctx, kv_len, "kv_len", a[4]), _ints(ctx, rows, "rows", n), n, _raw_stream(ctx, stream)))


def cp_pages_fork(ctx, pool, refcount, page_table, kv_len, parent, child, workspace, stream=None):
    """Rows child[i] become copies of rows parent[i]: full pages shared, the tokens of a partly filled last page copied in every layer."""
    a = _table_args(ctx, pool, refcount, page_table)
    n = parent.numel()
    _check(load().cp_pages_fork(*a, _ints(ctx, kv_len, "kv_len", a[4]), _ints(ctx, parent, "parent", n), _ints(ctx, child, "child", n), n,
                                *_workspace(ctx, workspace), _raw_stream(ctx, stream)))


def cp_pages_compact(ctx, pool, refcount, page_table, page_map, n_live, workspace, stream=None):
    """Move the pages in use to ids [0, n_live); page_map [num_pages] and n_live [1] (int32) receive the new ids and the count."""
    a = _table_args(ctx, pool, refcount, page_table)
    _check(load().cp_pages_compact(*a, _ints(ctx, page_map, "page_map", pool.num_pages), _ints(ctx, n_live, "n_live", 1), *_workspace(ctx, workspace),
                                   _raw_stream(ctx, stream)))


def cp_pages_copy(ctx, pool, src, dst, workspace, stream=None):
    """Page src[i] -> page dst[i] (int32 tensors) in every layer."""
    if _types is None:
        _torch_types()
    n = src.numel()
    _check(load().cp_pages_copy(ctx._h, _described(ctx, pool, cp_page_pool), _ints(ctx, src, "src", n), _ints(ctx, dst, "dst", n), n, *_workspace(ctx, workspace),
                                _raw_stream(ctx, stream)))
