"""ctypes binding of libcritiprefill.so: same names as the C ABI, argument marshalling only.

Tensors are torch CUDA tensors used purely as device buffers; every step of the path runs in the
library's HIP kernels.  There is no CPU fallback: a missing library or a non-zero status raises.
"""
from __future__ import annotations

import ctypes
import math
import os

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libcritiprefill.so")
_lib = None

CP_DTYPE_FP32, CP_DTYPE_BF16 = 0, 1
CP_CACHE_PLAIN, CP_CACHE_MXFP8, CP_CACHE_MXFP4 = 0, 1, 4
EXPORTS = ["critiprefill_list_len", "critiprefill_workspace_bytes", "critiprefill_estimate",
           "critiprefill_estimate_static", "critiprefill_select", "critiprefill_sparse_attn", "critiprefill_select_shared",
           "critiprefill_sparse_attn_shared", "critiprefill_dense_causal_attn",
           "critiprefill_norm_rope", "critiprefill_norm_rope_write", "critiprefill_cache_write", "critiprefill_cache_read",
           "critiprefill_paged_workspace_bytes", "critiprefill_paged_attn", "critiprefill_strerror", "critiprefill_version"]


class Params(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("seq_len", ctypes.c_int32), ("segment_size", ctypes.c_int32),
                ("block_size", ctypes.c_int32), ("budget_blocks", ctypes.c_int32), ("local_blocks", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("attn_scale", ctypes.c_float), ("score_scale", ctypes.c_float),
                ("alpha", ctypes.c_float), ("softmax_domain", ctypes.c_int32),
                ("q_stride", ctypes.c_int64 * 3), ("kv_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3)]


class CacheParams(ctypes.Structure):
    _fields_ = ([(x, ctypes.c_int32) for x in ("n_q_heads", "n_kv_heads", "head_dim", "dtype", "tokens", "cache_format", "page_size", "n_pages",
                                               "n_seqs", "max_pages", "max_q_len", "max_kv_len", "rotary_dim", "rotary_interleaved")]
                + [("norm_eps", ctypes.c_float), ("attn_scale", ctypes.c_float)]
                + [(x, ctypes.c_int64 * 2) for x in ("q_stride", "k_stride", "v_stride", "o_stride", "ko_stride")])


class CritiPrefillError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({strerror(status)})")


def lib_path() -> str:
    return _LIB_PATH


def load():
    """Load the shared library (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(f"{_LIB_PATH} not built: run `python -m paper_2409_12490_amd.build`")
    lib = ctypes.CDLL(_LIB_PATH)
    P = ctypes.POINTER(Params)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    lib.critiprefill_list_len.argtypes = [P]; lib.critiprefill_list_len.restype = ctypes.c_int32
    lib.critiprefill_workspace_bytes.argtypes = [P]; lib.critiprefill_workspace_bytes.restype = sz
    lib.critiprefill_estimate.argtypes = [P, vp, vp, vp, vp, vp, sz, vp]; lib.critiprefill_estimate.restype = ctypes.c_int
    lib.critiprefill_estimate_static.argtypes = [P, vp, vp, vp, vp, vp]; lib.critiprefill_estimate_static.restype = ctypes.c_int
    lib.critiprefill_select.argtypes = [P, vp, vp, vp, vp]; lib.critiprefill_select.restype = ctypes.c_int
    lib.critiprefill_sparse_attn.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp]; lib.critiprefill_sparse_attn.restype = ctypes.c_int
    lib.critiprefill_select_shared.argtypes = [P, vp, vp, vp, vp]; lib.critiprefill_select_shared.restype = ctypes.c_int
    lib.critiprefill_sparse_attn_shared.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp]; lib.critiprefill_sparse_attn_shared.restype = ctypes.c_int
    lib.critiprefill_dense_causal_attn.argtypes = [P, vp, vp, vp, vp, vp, vp]; lib.critiprefill_dense_causal_attn.restype = ctypes.c_int
    C = ctypes.POINTER(CacheParams)
    for name, pointers in (("norm_rope", 9), ("norm_rope_write", 14), ("cache_write", 8), ("cache_read", 8)):
        f = getattr(lib, "critiprefill_" + name)
        f.argtypes = [C] + [vp] * pointers; f.restype = ctypes.c_int
    lib.critiprefill_paged_workspace_bytes.argtypes = [C]; lib.critiprefill_paged_workspace_bytes.restype = sz
    lib.critiprefill_paged_attn.argtypes = [C] + [vp] * 11 + [sz, vp]; lib.critiprefill_paged_attn.restype = ctypes.c_int
    lib.critiprefill_strerror.argtypes = [ctypes.c_int]; lib.critiprefill_strerror.restype = ctypes.c_char_p
    lib.critiprefill_version.argtypes = []; lib.critiprefill_version.restype = ctypes.c_int
    _lib = lib
    return lib


def strerror(status: int) -> str:
    return load().critiprefill_strerror(status).decode()


def version() -> int:
    return load().critiprefill_version()


def make_params(q: torch.Tensor, k: torch.Tensor, segment_size: int, block_size: int, budget_blocks: int,
                local_blocks: int = 0, out: torch.Tensor | None = None, attn_scale: float = 0.0,
                score_scale: float = 0.0, alpha: float = 1.0, softmax_domain: int = 0) -> Params:
    """Fill the parameter block from tensor shapes/strides (q [B,Hq,n,d], k [B,Hkv,n,d])."""
    p = Params()
    p.batch, p.n_q_heads, p.seq_len, p.head_dim = q.shape[0], q.shape[1], q.shape[2], q.shape[3]
    p.n_kv_heads = k.shape[1]
    p.segment_size, p.block_size = segment_size, block_size
    p.budget_blocks, p.local_blocks = budget_blocks, local_blocks
    if q.dtype == torch.bfloat16:
        p.dtype = CP_DTYPE_BF16
    elif q.dtype == torch.float32:
        p.dtype = CP_DTYPE_FP32
    else:
        raise TypeError(f"unsupported dtype {q.dtype}")
    p.attn_scale, p.score_scale, p.alpha, p.softmax_domain = attn_scale, score_scale, alpha, softmax_domain
    if q.stride(3) != 1 or k.stride(3) != 1:
        raise ValueError("channel stride must be 1")
    for i in range(3):
        p.q_stride[i] = q.stride(i)
        p.kv_stride[i] = k.stride(i)
        p.o_stride[i] = (out if out is not None else q).stride(i)
    return p


def _ptr(t):
    return None if t is None else t.data_ptr()


# The current stream's handle straight from torch: torch.cuda.current_stream() builds a Stream object first (2.8 of the 7.3 us
# that a call of this module took on the host; the lookup below takes 0.1).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream(stream):
    if stream is None and _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream(_device())
    return (stream if stream is not None else torch.cuda.current_stream()).cuda_stream


def _check(status: int, where: str):
    if status != 0:
        raise CritiPrefillError(status, where)


def critiprefill_list_len(p: Params) -> int:
    return load().critiprefill_list_len(ctypes.byref(p))


def critiprefill_workspace_bytes(p: Params) -> int:
    return load().critiprefill_workspace_bytes(ctypes.byref(p))


def critiprefill_estimate(p, q, k, prev_scores, scores, workspace, stream=None):
    _check(load().critiprefill_estimate(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(prev_scores), _ptr(scores),
                                        _ptr(workspace), workspace.numel() * workspace.element_size(),
                                        _stream(stream)), "critiprefill_estimate")


def critiprefill_estimate_static(p, q, k, prev_scores, scores, stream=None):
    _check(load().critiprefill_estimate_static(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(prev_scores), _ptr(scores),
                                               _stream(stream)), "critiprefill_estimate_static")


def critiprefill_select(p, scores, block_idx, block_cnt, stream=None):
    _check(load().critiprefill_select(ctypes.byref(p), _ptr(scores), _ptr(block_idx), _ptr(block_cnt),
                                      _stream(stream)), "critiprefill_select")


def critiprefill_sparse_attn(p, q, k, v, block_idx, block_cnt, out, lse=None, stream=None):
    _check(load().critiprefill_sparse_attn(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(block_idx),
                                           _ptr(block_cnt), _ptr(out), _ptr(lse), _stream(stream)),
           "critiprefill_sparse_attn")


def critiprefill_select_shared(p, scores, block_idx, block_cnt, stream=None):
    _check(load().critiprefill_select_shared(ctypes.byref(p), _ptr(scores), _ptr(block_idx), _ptr(block_cnt),
                                             _stream(stream)), "critiprefill_select_shared")


def critiprefill_sparse_attn_shared(p, q, k, v, block_idx, block_cnt, out, lse=None, stream=None):
    _check(load().critiprefill_sparse_attn_shared(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(block_idx),
                                                  _ptr(block_cnt), _ptr(out), _ptr(lse), _stream(stream)),
           "critiprefill_sparse_attn_shared")


def critiprefill_dense_causal_attn(p, q, k, v, out, lse=None, stream=None):
    _check(load().critiprefill_dense_causal_attn(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse),
                                                 _stream(stream)), "critiprefill_dense_causal_attn")


# ---- the paged cache -----------------------------------------------------------------------------
def _dtype_code(dtype: torch.dtype) -> int:
    if dtype == torch.bfloat16:
        return CP_DTYPE_BF16
    if dtype == torch.float32:
        return CP_DTYPE_FP32
    raise TypeError(f"unsupported dtype {dtype}")


def make_cache_params(n_q_heads: int, n_kv_heads: int, dtype: torch.dtype, *, q=None, k=None, v=None, out=None, k_out=None, k_cache=None,
                      mxfp8: bool = False, page_table=None, max_q_len: int = 0, max_kv_len: int = 0, rotary_dim: int = 0, interleaved: bool = False,
                      norm_eps: float = 0.0, attn_scale: float = 0.0, mxfp4: bool = False) -> CacheParams:
    """Fill the parameter block from the tensors of a call: q, k, v, out (q_out or the attention's) and k_out are [tokens, heads, 128], each with
    strides of its own; k_cache [n_pages, n_kv_heads, page_size, 128], with mxfp4 64 bytes a row, says the pool's size, page_table [n_seqs, max_pages] the sequences."""
    p = CacheParams()
    p.n_q_heads, p.n_kv_heads, p.head_dim, p.dtype = n_q_heads, n_kv_heads, 128, _dtype_code(dtype)
    if mxfp8 and mxfp4:
        raise ValueError("mxfp8 and mxfp4: a cache has one format")
    p.cache_format = CP_CACHE_MXFP8 if mxfp8 else CP_CACHE_MXFP4 if mxfp4 else CP_CACHE_PLAIN
    tokens = None
    for t, heads, stride, name in ((q, n_q_heads, p.q_stride, "q"), (k, n_kv_heads, p.k_stride, "k"), (v, n_kv_heads, p.v_stride, "v"),
                                   (out, n_q_heads, p.o_stride, "out"), (k_out, n_kv_heads, p.ko_stride, "k_out")):
        if t is None:
            continue
        if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != 128 or (tokens is not None and t.shape[0] != tokens):
            raise ValueError(f"{name}: shape {tuple(t.shape)}, expected ({'tokens' if tokens is None else tokens}, {heads}, 128)")
        if t.dtype != dtype:
            raise TypeError(f"{name}: {t.dtype}, expected {dtype}")
        if t.stride(2) != 1:
            raise ValueError(f"{name}: channel stride must be 1")
        tokens = t.shape[0]
        for i in range(2):
            # the stride of an axis of one element is never used, and torch gives it any value
            stride[i] = t.stride(i) if t.shape[i] > 1 else max(128, heads * 128 if i == 0 else 128)
    p.tokens = tokens or 0
    if k_cache is not None:
        row = 64 if mxfp4 else 128
        if k_cache.dim() != 4 or k_cache.shape[1] != n_kv_heads or k_cache.shape[3] != row or not k_cache.is_contiguous():
            raise ValueError(f"k_cache: expected a contiguous [n_pages, {n_kv_heads}, page_size, {row}], got {tuple(k_cache.shape)}")
        if k_cache.dtype != (torch.uint8 if mxfp8 or mxfp4 else dtype):
            raise TypeError(f"k_cache: {k_cache.dtype}")
        p.n_pages, p.page_size = k_cache.shape[0], k_cache.shape[2]
    if page_table is not None:
        if page_table.dim() != 2 or not page_table.is_contiguous():
            raise ValueError("page_table: expected a contiguous [n_seqs, max_pages]")
        p.n_seqs, p.max_pages = page_table.shape
    p.max_q_len, p.max_kv_len, p.rotary_dim, p.rotary_interleaved = max_q_len, max_kv_len, rotary_dim, int(interleaved)
    p.norm_eps, p.attn_scale = norm_eps, attn_scale
    return p


def _refuse(t, dtype, least):
    raise ValueError(f"expected a contiguous tensor of {dtype} with {least} elements or more, got {t.dtype} {tuple(t.shape)}")


# Of all but q, k, v and the outputs, whose strides stand in the parameter block, the library sees only an address: type, size and contiguity are looked at here, at every
# call.  Of the others, that there are as many elements as the block says.  Written out, with no loop over arguments: a single token's operators take 4 us on the GPU.
_TYPES = {CP_DTYPE_FP32: torch.float32, CP_DTYPE_BF16: torch.bfloat16}


def _ints(t, least):
    if t.dtype is not torch.int32 or t.numel() < least or not t.is_contiguous():
        _refuse(t, torch.int32, least)
    return t.data_ptr()


def _weight(t, dtype):
    if t.dtype is not dtype or t.numel() != 128 or not t.is_contiguous():
        raise ValueError(f"weight: expected 128 contiguous elements of {dtype}, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _few(tokens, *tensors):
    raise ValueError(f"the parameter block says {tokens} tokens, got {' '.join(str(tuple(t.shape)) for t in tensors)}")


def _pool(p, k_cache, v_cache, k_scale, v_scale):
    """The addresses of the pool's four tensors, which the library takes to be as large as n_pages says."""
    rows = p.n_pages * p.n_kv_heads * p.page_size
    scaled = p.cache_format != CP_CACHE_PLAIN
    size = rows * (64 if p.cache_format == CP_CACHE_MXFP4 else 128)
    dtype = torch.uint8 if scaled else _TYPES.get(p.dtype)
    if k_cache.dtype is not dtype or k_cache.numel() < size or not k_cache.is_contiguous():
        _refuse(k_cache, dtype, size)
    if v_cache.dtype is not dtype or v_cache.numel() < size or not v_cache.is_contiguous():
        _refuse(v_cache, dtype, size)
    if not scaled or k_scale is None or v_scale is None:                  # not read, or refused by the library
        return k_cache.data_ptr(), v_cache.data_ptr(), _ptr(k_scale), _ptr(v_scale)
    if k_scale.dtype is not torch.uint8 or k_scale.numel() < 4 * rows or not k_scale.is_contiguous():
        _refuse(k_scale, torch.uint8, 4 * rows)
    if v_scale.dtype is not torch.uint8 or v_scale.numel() < 4 * rows or not v_scale.is_contiguous():
        _refuse(v_scale, torch.uint8, 4 * rows)
    return k_cache.data_ptr(), v_cache.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr()


def _angles(p, inv_freq, positions):
    if p.rotary_dim == 0:
        return None, None
    least = p.rotary_dim // 2
    if inv_freq is None or positions is None:
        return _ptr(inv_freq), _ptr(positions)
    if inv_freq.dtype is not torch.float64 or inv_freq.numel() < least or not inv_freq.is_contiguous():
        _refuse(inv_freq, torch.float64, least)
    return inv_freq.data_ptr(), _ints(positions, p.tokens)


def critiprefill_norm_rope(p, q, k, q_weight, k_weight, inv_freq, positions, q_out, k_out, stream=None):
    freq, pos = _angles(p, inv_freq, positions)
    dtype, channels = _TYPES.get(p.dtype), p.tokens * 128
    least_q, least_k = channels * p.n_q_heads, channels * p.n_kv_heads
    if q.numel() < least_q or k.numel() < least_k or q_out.numel() < least_q or k_out.numel() < least_k:
        _few(p.tokens, q, k, q_out, k_out)
    _check((_lib or load()).critiprefill_norm_rope(
        p, q.data_ptr(), k.data_ptr(), None if q_weight is None else _weight(q_weight, dtype), None if k_weight is None else _weight(k_weight, dtype), freq, pos,
        q_out.data_ptr(), k_out.data_ptr(), _stream(stream)), "critiprefill_norm_rope")


def critiprefill_norm_rope_write(p, q, k, v, q_weight, k_weight, inv_freq, positions, slots, q_out, k_cache, v_cache, k_scale=None, v_scale=None,
                                 stream=None):
    freq, pos = _angles(p, inv_freq, positions)
    dtype, tokens = _TYPES.get(p.dtype), p.tokens
    least_q, least_k = tokens * 128 * p.n_q_heads, tokens * 128 * p.n_kv_heads
    if q.numel() < least_q or k.numel() < least_k or v.numel() < least_k or q_out.numel() < least_q:
        _few(tokens, q, k, v, q_out)
    _check((_lib or load()).critiprefill_norm_rope_write(
        p, q.data_ptr(), k.data_ptr(), v.data_ptr(), None if q_weight is None else _weight(q_weight, dtype), None if k_weight is None else _weight(k_weight, dtype),
        freq, pos, _ints(slots, tokens), q_out.data_ptr(), *_pool(p, k_cache, v_cache, k_scale, v_scale), _stream(stream)), "critiprefill_norm_rope_write")


def critiprefill_cache_write(p, k, v, slots, k_cache, v_cache, k_scale=None, v_scale=None, stream=None):
    tokens = p.tokens
    least = tokens * 128 * p.n_kv_heads
    if k.numel() < least or v.numel() < least:
        _few(tokens, k, v)
    _check((_lib or load()).critiprefill_cache_write(
        p, k.data_ptr(), v.data_ptr(), _ints(slots, tokens), *_pool(p, k_cache, v_cache, k_scale, v_scale), _stream(stream)), "critiprefill_cache_write")


def critiprefill_cache_read(p, slots, k_cache, v_cache, k_scale, v_scale, k, v, stream=None):
    tokens = p.tokens
    least = tokens * 128 * p.n_kv_heads
    if k.numel() < least or v.numel() < least:
        _few(tokens, k, v)
    _check((_lib or load()).critiprefill_cache_read(
        p, _ints(slots, tokens), *_pool(p, k_cache, v_cache, k_scale, v_scale), k.data_ptr(), v.data_ptr(), _stream(stream)), "critiprefill_cache_read")


def critiprefill_paged_workspace_bytes(p: CacheParams) -> int:
    return load().critiprefill_paged_workspace_bytes(ctypes.byref(p))


def critiprefill_paged_attn(p, q, k_cache, v_cache, k_scale, v_scale, page_table, q_start, kv_len, out, lse, workspace, stream=None):
    seqs = p.n_seqs
    rows = p.tokens * p.n_q_heads
    if q.numel() < rows * 128 or out.numel() < rows * 128:
        _few(p.tokens, q, out)
    if lse is not None and (lse.dtype is not torch.float32 or lse.numel() < rows or not lse.is_contiguous()):
        _refuse(lse, torch.float32, rows)
    _check((_lib or load()).critiprefill_paged_attn(
        p, q.data_ptr(), *_pool(p, k_cache, v_cache, k_scale, v_scale), _ints(page_table, seqs * p.max_pages), _ints(q_start, seqs + 1), _ints(kv_len, seqs),
        out.data_ptr(), None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
        _stream(stream)), "critiprefill_paged_attn")


# ---- buffer helpers (device memory only; no arithmetic) -----------------------------------------
def n_segments(p: Params) -> int:
    return -(-p.seq_len // p.segment_size)


def n_blocks(p: Params) -> int:
    return -(-p.seq_len // p.block_size)


def alloc_scores(p: Params, device="cuda") -> torch.Tensor:
    return torch.empty((p.batch, p.n_q_heads, n_segments(p), n_blocks(p)), dtype=torch.float32, device=device)


def alloc_lists(p: Params, device="cuda"):
    ll = critiprefill_list_len(p)
    idx = torch.empty((p.batch, p.n_q_heads, n_segments(p), ll), dtype=torch.int32, device=device)
    cnt = torch.empty((p.batch, p.n_q_heads, n_segments(p)), dtype=torch.int32, device=device)
    return idx, cnt


def alloc_shared_lists(p: Params, device="cuda"):
    """Lists of critiprefill_select_shared: one per (batch, KV head, segment)."""
    ll = critiprefill_list_len(p)
    idx = torch.empty((p.batch, p.n_kv_heads, n_segments(p), ll), dtype=torch.int32, device=device)
    cnt = torch.empty((p.batch, p.n_kv_heads, n_segments(p)), dtype=torch.int32, device=device)
    return idx, cnt


def alloc_workspace(p: Params, device="cuda") -> torch.Tensor:
    return torch.empty((max(16, critiprefill_workspace_bytes(p)),), dtype=torch.uint8, device=device)


def alloc_cache(n_pages: int, n_kv_heads: int, page_size: int, dtype: torch.dtype = torch.bfloat16, mxfp8: bool = False, device="cuda", mxfp4: bool = False):
    """(k_cache, v_cache, k_scale, v_scale) of a pool of pages; the scales are None without mxfp8 and mxfp4."""
    if mxfp8 and mxfp4:
        raise ValueError("mxfp8 and mxfp4: a cache has one format")
    shape, scaled = (n_pages, n_kv_heads, page_size), mxfp8 or mxfp4
    caches = [torch.empty((*shape, 64 if mxfp4 else 128), dtype=torch.uint8 if scaled else dtype, device=device) for _ in range(2)]
    scales = [torch.empty((*shape, 4), dtype=torch.uint8, device=device) if scaled else None for _ in range(2)]
    return (*caches, *scales)


def alloc_paged_workspace(p: CacheParams, device="cuda") -> torch.Tensor:
    return torch.empty((max(16, critiprefill_paged_workspace_bytes(p)),), dtype=torch.uint8, device=device)


def rotary_frequencies(rotary_dim: int = 128, base: float = 500000.0, device="cuda") -> torch.Tensor:
    """inv_freq of critiprefill_norm_rope for the usual base^(-2c / rotary_dim)."""
    return base ** (-torch.arange(rotary_dim // 2, dtype=torch.float64, device=device) * 2 / rotary_dim)
