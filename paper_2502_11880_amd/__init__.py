"""Ternary-weight x int8-activation mpGEMM for AMD MI355X (gfx950), after Bitnet.cpp (arXiv 2502.11880).

This package is a thin ctypes binding over the C ABI in ``include/bitnet_mi355x.h``: each function
below has the name of the C entry point it calls, checks and marshals its torch arguments (device,
dtype, contiguity) and raises ``BitnetError`` on a non-OK status.  All arithmetic runs in the HIP
kernels of ``libbitnet_mi355x.so``; if that library has not been built, every call raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
import threading

LIB_NAME = "libbitnet_mi355x.so"
LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), LIB_NAME)

BITNET_LAYOUT_I2S = 0
BITNET_LAYOUT_TL2 = 1
BITNET_LAYOUT_TL1 = 2
BITNET_LAYOUT_C4G2 = 3
BITNET_LAYOUT_C5G2 = 4
BITNET_LAYOUT_C3G5 = 5
BITNET_LAYOUT_TL2_0 = 6
BITNET_LAYOUT_TL1_0 = 7
LAYOUTS = {"i2s": BITNET_LAYOUT_I2S, "tl2": BITNET_LAYOUT_TL2, "tl1": BITNET_LAYOUT_TL1, "c4g2": BITNET_LAYOUT_C4G2,
           "c5g2": BITNET_LAYOUT_C5G2, "c3g5": BITNET_LAYOUT_C3G5, "tl2_0": BITNET_LAYOUT_TL2_0,
           "tl1_0": BITNET_LAYOUT_TL1_0}
INT_LAYOUTS = ("c4g2", "c5g2", "c3g5")

BITNET_OK = 0
STATUS_NAMES = {0: "BITNET_OK", 1: "BITNET_E_INVALID", 2: "BITNET_E_SHAPE", 3: "BITNET_E_ALIGN",
                4: "BITNET_E_LAYOUT", 5: "BITNET_E_WORKSPACE", 6: "BITNET_E_HIP"}

# (name, restype, argtypes) of every exported entry point, in header order
_SIGNATURES = [
    ("bitnet_packed_bytes", ctypes.c_size_t, [ctypes.c_int, ctypes.c_int64, ctypes.c_int64]),
    ("bitnet_pack_workspace_bytes", ctypes.c_size_t, [ctypes.c_int64, ctypes.c_int64]),
    ("bitnet_pack_weights", ctypes.c_int,
     [ctypes.c_int, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t,
      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    ("bitnet_pack_int_weights", ctypes.c_int,
     [ctypes.c_int, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    ("bitnet_quantize_act", ctypes.c_int,
     [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
      ctypes.c_void_p]),
    ("bitnet_mpgemm_workspace_bytes", ctypes.c_size_t, [ctypes.c_int, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64]),
    ("bitnet_mpgemm", ctypes.c_int,
     [ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p,
      ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    ("bitnet_mpgemm_noalloc", ctypes.c_int,
     [ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p,
      ctypes.c_void_p]),
    ("bitnet_mpgemm_fused_workspace_bytes", ctypes.c_size_t,
     [ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64]),
    ("bitnet_mpgemm_fused", ctypes.c_int,
     [ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
      ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
      ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    ("bitnet_elut_tables", ctypes.c_int,
     [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    ("bitnet_kv_page_bytes", ctypes.c_size_t,
     [ctypes.c_int, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int]),
    ("bitnet_kv_append", ctypes.c_int,
     [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p]),
    ("bitnet_attn_decode_workspace_bytes", ctypes.c_size_t, [ctypes.c_int64] * 8),
    ("bitnet_attn_decode", ctypes.c_int,
     [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_int64, ctypes.c_int64,
      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    ("bitnet_attn_prefill_workspace_bytes", ctypes.c_size_t, [ctypes.c_int] * 2 + [ctypes.c_int64] * 9),
    ("bitnet_attn_prefill", ctypes.c_int,
     [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_float,
      ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    ("bitnet_kv_workspace_bytes", ctypes.c_size_t, [ctypes.c_int64, ctypes.c_int64]),
    ("bitnet_kv_copy_pages", ctypes.c_int,
     [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p]),
    ("bitnet_kv_reserve", ctypes.c_int,
     [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p,
      ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    ("bitnet_kv_fork", ctypes.c_int,
     [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    ("bitnet_kv_free", ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p]),
    ("bitnet_kv_trim", ctypes.c_int,
     [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p]),
    ("bitnet_kv_compact", ctypes.c_int,
     [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    ("bitnet_status_string", ctypes.c_char_p, [ctypes.c_int]),
    ("bitnet_last_error", ctypes.c_char_p, []),
]

_lock = threading.Lock()
_handle = None


class BitnetError(RuntimeError):
    def __init__(self, fn: str, status: int, detail: str):
        self.status = status
        super().__init__(f"{fn} failed: {STATUS_NAMES.get(status, status)}: {detail}")


def lib():
    """The loaded C library (loads it on first use; raises if it is not built)."""
    global _handle
    if _handle is not None:
        return _handle
    with _lock:
        if _handle is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(f"{LIB_NAME} is not built; run `python -m paper_2502_11880_amd.build` "
                                   "(or __graft_entry__.build()) first")
            h = ctypes.CDLL(LIB_PATH)
            for name, res, args in _SIGNATURES:
                fn = getattr(h, name)
                fn.restype = res
                fn.argtypes = args
            _handle = h
        return _handle


def _check(fn: str, status: int) -> None:
    if status != BITNET_OK:
        detail = lib().bitnet_last_error().decode(errors="replace")
        raise BitnetError(fn, status, detail)


def _layout(layout) -> int:
    if isinstance(layout, str):
        return LAYOUTS[layout.lower()]
    return int(layout)


def _ptr(t, name, dtype=None, device=True):
    if t is None:
        return None
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if device and not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


@functools.lru_cache(maxsize=None)
def _current_stream():
    """A call that returns the current stream's handle (building a torch.cuda.Stream for it takes 2.7 us, a third of a call)."""
    import torch
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is None or device is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    torch.cuda.init()
    return lambda: raw(device())


def _stream(stream):
    if stream is None:
        return _current_stream()()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# ------------------------------------------------------------------------------------------------
# Size queries (pure host functions)
# ------------------------------------------------------------------------------------------------
def bitnet_packed_bytes(layout, N: int, K: int) -> int:
    return int(lib().bitnet_packed_bytes(_layout(layout), N, K))


def bitnet_pack_workspace_bytes(N: int, K: int) -> int:
    return int(lib().bitnet_pack_workspace_bytes(N, K))


def bitnet_mpgemm_workspace_bytes(layout, M: int, N: int, K: int) -> int:
    return int(lib().bitnet_mpgemm_workspace_bytes(_layout(layout), M, N, K))


# ------------------------------------------------------------------------------------------------
# Entry points
# ------------------------------------------------------------------------------------------------
def bitnet_pack_weights(layout, W, packed, w_scale, ws, stream=None) -> None:
    """Ternarise and pack W (fp32 [N, K], device) into `packed` (uint8) and `w_scale` (fp32 [1])."""
    import torch
    N, K = W.shape
    st = lib().bitnet_pack_weights(_layout(layout), _ptr(W, "W", torch.float32), N, K,
                                   _ptr(packed, "packed", torch.uint8), packed.numel(),
                                   _ptr(w_scale, "w_scale", torch.float32), _ptr(ws, "ws"),
                                   ws.numel() * ws.element_size(), _stream(stream))
    _check("bitnet_pack_weights", st)


def bitnet_pack_int_weights(layout, Wq, packed, stream=None) -> None:
    """Pack integer weights Wq (int8 [N, K], device) for an integer-weight layout (c4g2, c5g2, c3g5)."""
    import torch
    N, K = Wq.shape
    st = lib().bitnet_pack_int_weights(_layout(layout), _ptr(Wq, "Wq", torch.int8), N, K,
                                       _ptr(packed, "packed", torch.uint8), packed.numel(), _stream(stream))
    _check("bitnet_pack_int_weights", st)


def bitnet_quantize_act(x, xq, x_scale, x_rowsum=None, stream=None) -> None:
    """Per-token absmax int8 quantisation of x (fp32 [M, K], device) into xq (int8), x_scale (fp32 [M]) and,
    optionally, x_rowsum (int32 [M])."""
    import torch
    M, K = x.shape
    st = lib().bitnet_quantize_act(_ptr(x, "x", torch.float32), M, K, _ptr(xq, "xq", torch.int8),
                                   _ptr(x_scale, "x_scale", torch.float32), _ptr(x_rowsum, "x_rowsum", torch.int32),
                                   _stream(stream))
    _check("bitnet_quantize_act", st)


def bitnet_mpgemm(layout, packed, w_scale, N: int, K: int, xq, x_scale, y, acc=None, ws=None, stream=None,
                  x_rowsum=None) -> None:
    """y = dequant(xq @ t^T) for the packed ternary weight; optionally the exact int32 accumulators."""
    import torch
    M = xq.shape[0]
    ws_ptr = _ptr(ws, "ws") if ws is not None else None
    ws_bytes = ws.numel() * ws.element_size() if ws is not None else 0
    st = lib().bitnet_mpgemm(_layout(layout), _ptr(packed, "packed", torch.uint8), packed.numel(),
                             _ptr(w_scale, "w_scale", torch.float32), N, K, _ptr(xq, "xq", torch.int8),
                             _ptr(x_scale, "x_scale", torch.float32), _ptr(x_rowsum, "x_rowsum", torch.int32), M,
                             _ptr(y, "y", torch.float32),
                             _ptr(acc, "acc", torch.int32), ws_ptr, ws_bytes, _stream(stream))
    _check("bitnet_mpgemm", st)


NOALLOC_SCRATCH_BYTES = 32 << 20     # BITNET_NOALLOC_SCRATCH_BYTES


def bitnet_mpgemm_noalloc(layout, packed, w_scale, N: int, K: int, xq, x_scale, y, acc=None, stream=None,
                          x_rowsum=None) -> None:
    """bitnet_mpgemm with its workspace taken from the library's static per-GPU scratch (no allocation)."""
    import torch
    M = xq.shape[0]
    st = lib().bitnet_mpgemm_noalloc(_layout(layout), _ptr(packed, "packed", torch.uint8), packed.numel(),
                                     _ptr(w_scale, "w_scale", torch.float32), N, K, _ptr(xq, "xq", torch.int8),
                                     _ptr(x_scale, "x_scale", torch.float32),
                                     _ptr(x_rowsum, "x_rowsum", torch.int32), M, _ptr(y, "y", torch.float32),
                                     _ptr(acc, "acc", torch.int32), _stream(stream))
    _check("bitnet_mpgemm_noalloc", st)


def bitnet_mpgemm_fused_workspace_bytes(layout, Ns, K: int, M: int) -> int:
    """Workspace bytes with which bitnet_mpgemm_fused runs every K split it can use for weights of rows Ns (a list)
    at M tokens: at least the largest single-weight workspace."""
    arr = (ctypes.c_int64 * len(Ns))(*Ns)
    return int(lib().bitnet_mpgemm_fused_workspace_bytes(_layout(layout), len(Ns), arr, K, M))


class FusedArgs:
    """Host arrays for bitnet_mpgemm_fused, built once so repeated calls only pass pointers."""

    def __init__(self, packed, w_scales, ys):
        import torch
        n = len(packed)
        self.n = n
        self.packed = (ctypes.c_void_p * n)(*[_ptr(p, "packed", torch.uint8) for p in packed])
        self.packed_bytes = (ctypes.c_size_t * n)(*[p.numel() for p in packed])
        self.w_scale = (ctypes.c_void_p * n)(*[_ptr(w, "w_scale", torch.float32) for w in w_scales])
        self.N = (ctypes.c_int64 * n)(*[y.shape[1] for y in ys])
        self.y = (ctypes.c_void_p * n)(*[_ptr(y, "y", torch.float32) for y in ys])
        self._keep = (list(packed), list(w_scales), list(ys))


def bitnet_mpgemm_fused(layout, packed, w_scales, x, xq, x_scale, x_rowsum, ys, ws=None, stream=None,
                        args: FusedArgs = None) -> None:
    """Quantise x (fp32 [M, K]) and multiply it by every packed weight (lists of equal length) in one call.
    With x None, xq / x_scale / x_rowsum already hold the quantised activation and only the products run."""
    import torch
    M, K = (x if x is not None else xq).shape
    a = args if args is not None else FusedArgs(packed, w_scales, ys)
    if a.n < 1:
        raise ValueError("bitnet_mpgemm_fused needs at least one weight")
    ws_ptr = _ptr(ws, "ws") if ws is not None else None
    ws_bytes = ws.numel() * ws.element_size() if ws is not None else 0
    st = lib().bitnet_mpgemm_fused(_layout(layout), a.n, a.packed, a.packed_bytes, a.w_scale, a.N, K,
                                   _ptr(x, "x", torch.float32) if x is not None else None, M,
                                   _ptr(xq, "xq", torch.int8),
                                   _ptr(x_scale, "x_scale", torch.float32), _ptr(x_rowsum, "x_rowsum", torch.int32),
                                   a.y, ws_ptr, ws_bytes, _stream(stream))
    _check("bitnet_mpgemm_fused", st)


def bitnet_elut_tables(xq, lut, lut1=None, stream=None) -> None:
    """TL2 activation tables of xq (int8 [M, K], device) into lut (int16 [M, ThreeK/3, 16]) and lut1."""
    import torch
    M, K = xq.shape
    st = lib().bitnet_elut_tables(_ptr(xq, "xq", torch.int8), M, K, _ptr(lut, "lut", torch.int16),
                                  _ptr(lut1, "lut1", torch.int16), _stream(stream))
    _check("bitnet_elut_tables", st)


# ------------------------------------------------------------------------------------------------
# The paged key-value cache and its attention
# ------------------------------------------------------------------------------------------------
BITNET_DTYPE_F32 = 0
BITNET_DTYPE_BF16 = 1
BITNET_DTYPE_F16 = 2


class _KvCache(ctypes.Structure):          # bitnet_kv_cache
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("table", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("n_pages", ctypes.c_int64), ("n_seqs", ctypes.c_int64), ("max_pages", ctypes.c_int64),
                ("page_size", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class _KvPool(ctypes.Structure):           # bitnet_kv_pool
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("n_layers", ctypes.c_int64), ("n_pages", ctypes.c_int64),
                ("k_page_bytes", ctypes.c_int64), ("v_page_bytes", ctypes.c_int64)]


class _KvTables(ctypes.Structure):         # bitnet_kv_tables
    _fields_ = [("table", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("refs", ctypes.c_void_p),
                ("n_seqs", ctypes.c_int64), ("max_pages", ctypes.c_int64), ("n_pages", ctypes.c_int64)]


@functools.lru_cache(maxsize=None)
def _types():
    """(int32, the value of bitnet_dtype of every type it has)."""
    import torch
    return torch.int32, {torch.float32: BITNET_DTYPE_F32, torch.bfloat16: BITNET_DTYPE_BF16, torch.float16: BITNET_DTYPE_F16}


def _dtype(t, name) -> int:
    d = _types()[1].get(t.dtype)
    if d is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return d


def _cache(k_cache, v_cache, table, kv_len):
    """The C description of one layer's cache, from tensors k_cache [n_pages, Hkv, ceil(D / 8), page_size, 8] and
    v_cache [n_pages, Hkv, page_size / 8, D, 8] (bfloat16 or float16), table int32 [n_seqs, max_pages] and kv_len int32
    [n_seqs]."""
    ks, vs, ts = k_cache.shape, v_cache.shape, table.shape
    if len(ks) != 5 or len(vs) != 5 or len(ts) != 2:
        raise ValueError("k_cache and v_cache must have 5 dimensions and table 2")
    pages, heads, chunks, ps, eight = ks
    dim = vs[3]
    if eight != 8 or chunks != -(-dim // 8) or vs != (pages, heads, ps // 8, dim, 8):
        raise ValueError(f"k_cache {tuple(ks)} and v_cache {tuple(vs)} are not "
                         "[pages, heads, ceil(dim / 8), page_size, 8] and [pages, heads, page_size / 8, dim, 8]")
    if v_cache.dtype is not k_cache.dtype:
        raise TypeError(f"v_cache must be {k_cache.dtype}, got {v_cache.dtype}")
    seqs, width = ts
    if kv_len.numel() != seqs:
        raise ValueError(f"kv_len must have one entry for each of the {seqs} rows of table, got {kv_len.numel()}")
    i32 = _types()[0]
    return _KvCache(_ptr(k_cache, "k_cache"), _ptr(v_cache, "v_cache"), _ptr(table, "table", i32),
                    _ptr(kv_len, "kv_len", i32), pages, seqs, width, ps, heads, dim, _dtype(k_cache, "k_cache"))


def _q_start(q_start, seqs):
    if q_start.numel() != seqs + 1:
        raise ValueError(f"q_start must have {seqs + 1} entries, got {q_start.numel()}")
    return _ptr(q_start, "q_start", _types()[0])


def _rows(t, name, heads_dim):
    """Tokens of a [tokens, heads, dim] or [tokens, heads * dim] tensor."""
    n = t.shape[0]
    if t.numel() != n * heads_dim:
        raise ValueError(f"{name} {tuple(t.shape)} must have rows of {heads_dim} values")
    return n


def bitnet_kv_page_bytes(dtype: int, page_size: int, n_kv_heads: int, head_dim: int, values: bool) -> int:
    return int(lib().bitnet_kv_page_bytes(dtype, page_size, n_kv_heads, head_dim, 1 if values else 0))


def bitnet_kv_append(k, v, q_start, k_cache, v_cache, table, kv_len, stream=None) -> None:
    """Write k and v ([tokens, Hkv * D], float32 or the cache's type) into the pages of their sequences: tokens
    q_start[s] .. q_start[s + 1] - 1 become the last ones of sequence s, whose kv_len counts them already.  q_start
    None: one token a sequence."""
    c = _cache(k_cache, v_cache, table, kv_len)
    n = _rows(k, "k", c.n_kv_heads * c.head_dim)
    if v.numel() != k.numel() or v.dtype != k.dtype:
        raise ValueError("k and v must have one size and type")
    st = lib().bitnet_kv_append(ctypes.byref(c), _ptr(k, "k"), _ptr(v, "v"), _dtype(k, "k"),
                                None if q_start is None else _q_start(q_start, c.n_seqs), n, _stream(stream))
    _check("bitnet_kv_append", st)


def bitnet_attn_decode_workspace_bytes(n_seqs: int, n_heads: int, n_kv_heads: int, head_dim: int, page_size: int,
                                       max_pages: int, window: int = 0, n_sink: int = 0) -> int:
    return int(lib().bitnet_attn_decode_workspace_bytes(n_seqs, n_heads, n_kv_heads, head_dim, page_size, max_pages,
                                                        window, n_sink))


def _heads(q, out, c, n):
    if out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError("out must have q's size and type")
    if n == 0:
        return c.n_kv_heads
    heads, rest = divmod(q.numel(), n * c.head_dim)
    if rest:
        raise ValueError(f"q {tuple(q.shape)} must have rows of whole heads of {c.head_dim}")
    return heads


def bitnet_attn_decode(q, k_cache, v_cache, table, kv_len, out, scale: float, window: int = 0, n_sink: int = 0, ws=None,
                       stream=None) -> None:
    """out[s] = attention of q[s] ([n_seqs, H * D], float32 or the cache's type) over the kv_len[s] cached tokens, or
    with window > 0 over the last `window` and the first `n_sink` of them."""
    c = _cache(k_cache, v_cache, table, kv_len)
    if q.shape[0] != c.n_seqs:
        raise ValueError(f"q must have one row for each of the {c.n_seqs} sequences, got {q.shape[0]}")
    st = lib().bitnet_attn_decode(ctypes.byref(c), _ptr(q, "q"), _dtype(q, "q"), _heads(q, out, c, c.n_seqs), scale, window,
                                  n_sink, _ptr(out, "out"), _ptr(ws, "ws"),
                                  0 if ws is None else ws.numel() * ws.element_size(), _stream(stream))
    _check("bitnet_attn_decode", st)


def bitnet_attn_prefill_workspace_bytes(cache_dtype: int, dtype: int, n_seqs: int, n_tokens: int, n_heads: int,
                                        n_kv_heads: int, head_dim: int, page_size: int, max_pages: int, window: int = 0,
                                        n_sink: int = 0) -> int:
    return int(lib().bitnet_attn_prefill_workspace_bytes(cache_dtype, dtype, n_seqs, n_tokens, n_heads, n_kv_heads, head_dim,
                                                         page_size, max_pages, window, n_sink))


def bitnet_attn_prefill(q, q_start, k_cache, v_cache, table, kv_len, out, scale: float, window: int = 0, n_sink: int = 0,
                        ws=None, stream=None) -> None:
    """Causal attention of the new tokens q ([tokens, H * D], float32 or the cache's type), which the cache already holds:
    rows q_start[s] .. q_start[s + 1] - 1 are the last tokens of sequence s.  ws (optional): a workspace of
    bitnet_attn_prefill_workspace_bytes, with which few queries split their keys; where there is none and the call goes to
    the current stream, one is taken from torch's allocator."""
    c = _cache(k_cache, v_cache, table, kv_len)
    n = q.shape[0]
    heads, dtype = _heads(q, out, c, n), _dtype(q, "q")
    if ws is None and stream is None:
        need = lib().bitnet_attn_prefill_workspace_bytes(c.dtype, dtype, c.n_seqs, n, heads, c.n_kv_heads, c.head_dim,
                                                         c.page_size, c.max_pages, window, n_sink)
        if need:
            import torch
            ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    st = lib().bitnet_attn_prefill(ctypes.byref(c), _ptr(q, "q"), dtype, heads, _q_start(q_start, c.n_seqs), n, scale, window,
                                   n_sink, _ptr(out, "out"), _ptr(ws, "ws"),
                                   0 if ws is None else ws.numel() * ws.element_size(), _stream(stream))
    _check("bitnet_attn_prefill", st)


def _pool(k_pool, v_pool):
    """The C description of the caches of all layers: k_pool [layers, *k_cache.shape], v_pool [layers, *v_cache.shape]."""
    if k_pool.dim() != 6 or v_pool.dim() != 6 or v_pool.shape[:3] != k_pool.shape[:3]:
        raise ValueError("k_pool and v_pool must be [layers, n_pages, heads, ...] with 6 dimensions")
    layers, pages = k_pool.shape[:2]
    n = max(1, layers * pages)
    return _KvPool(_ptr(k_pool, "k_pool"), _ptr(v_pool, "v_pool"), layers, pages,
                   k_pool.numel() // n * k_pool.element_size(), v_pool.numel() // n * v_pool.element_size())


def _tables(table, kv_len, refs):
    i32 = _types()[0]
    if table.dim() != 2 or (kv_len is not None and kv_len.numel() != table.shape[0]):
        raise ValueError("table must be [n_seqs, max_pages] and kv_len [n_seqs]")
    return _KvTables(_ptr(table, "table", i32), _ptr(kv_len, "kv_len", i32), _ptr(refs, "refs", i32), table.shape[0], table.shape[1], refs.numel())


def _list(t, name, n=None):
    if n is not None and t.numel() != n:
        raise ValueError(f"{name} must have {n} entries, got {t.numel()}")
    return _ptr(t, name, _types()[0])


def bitnet_kv_workspace_bytes(n_pages: int, n_seqs: int) -> int:
    return int(lib().bitnet_kv_workspace_bytes(n_pages, n_seqs))


def bitnet_kv_copy_pages(k_pool, v_pool, src, dst, stream=None) -> None:
    """Copy page src[i] to page dst[i] (int32 device lists) in every layer."""
    p = _pool(k_pool, v_pool)
    n = src.numel()
    st = lib().bitnet_kv_copy_pages(ctypes.byref(p), _list(src, "src"), _list(dst, "dst", n), n, _stream(stream))
    _check("bitnet_kv_copy_pages", st)


def bitnet_kv_reserve(table, kv_len, refs, seqs, n_new, page_size: int, n_short, ws, stream=None) -> None:
    """Pages for n_new[i] more tokens of sequence seqs[i], counted in kv_len; n_short (int32 [1]) receives the number of
    sequences that could not have them and stayed as they were.  In the list's order: once the free pages do not suffice for
    one, later ones are only served where their tokens need no new page."""
    t = _tables(table, kv_len, refs)
    n = seqs.numel()
    st = lib().bitnet_kv_reserve(ctypes.byref(t), _list(seqs, "seqs"), _list(n_new, "n_new", n), n, page_size,
                                 _list(n_short, "n_short", 1), _ptr(ws, "ws"), ws.numel() * ws.element_size(),
                                 _stream(stream))
    _check("bitnet_kv_reserve", st)


def bitnet_kv_fork(k_pool, v_pool, table, kv_len, refs, parents, children, n_short, ws, stream=None) -> None:
    """Sequence children[i] becomes a copy of parents[i]: full pages shared, a last partial page copied in every layer."""
    p = _pool(k_pool, v_pool)
    t = _tables(table, kv_len, refs)
    n = children.numel()
    st = lib().bitnet_kv_fork(ctypes.byref(p), ctypes.byref(t), _list(parents, "parents", n), _list(children, "children"),
                              n, k_pool.shape[4], _list(n_short, "n_short", 1), _ptr(ws, "ws"),
                              ws.numel() * ws.element_size(), _stream(stream))
    _check("bitnet_kv_fork", st)


def bitnet_kv_free(table, kv_len, refs, seqs, stream=None) -> None:
    """Give back the pages of the listed sequences."""
    t = _tables(table, kv_len, refs)
    st = lib().bitnet_kv_free(ctypes.byref(t), _list(seqs, "seqs"), seqs.numel(), _stream(stream))
    _check("bitnet_kv_free", st)


def bitnet_kv_trim(table, kv_len, refs, seqs, page_size: int, window: int, n_sink: int = 0, stream=None) -> None:
    """Give back the listed sequences' pages that lie wholly behind the window of their next token and past the sinks."""
    t = _tables(table, kv_len, refs)
    st = lib().bitnet_kv_trim(ctypes.byref(t), _list(seqs, "seqs"), seqs.numel(), page_size, window, n_sink,
                              _stream(stream))
    _check("bitnet_kv_trim", st)


def bitnet_kv_compact(k_pool, v_pool, table, refs, n_live, ws, stream=None) -> None:
    """Move the live pages to the lowest numbers, in every layer; n_live (int32 [1]) receives their count."""
    p = _pool(k_pool, v_pool)
    t = _tables(table, None, refs)
    st = lib().bitnet_kv_compact(ctypes.byref(p), ctypes.byref(t), _list(n_live, "n_live", 1), _ptr(ws, "ws"),
                                 ws.numel() * ws.element_size(), _stream(stream))
    _check("bitnet_kv_compact", st)


def bitnet_status_string(status: int) -> str:
    return lib().bitnet_status_string(status).decode()


def bitnet_last_error() -> str:
    return lib().bitnet_last_error().decode(errors="replace")
