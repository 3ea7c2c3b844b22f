"""Thin ctypes binding of librsa.so: argument marshalling only.

The entry points carry the names of the C-ABI (include/rsa.h). Tensors are torch CUDA
(ROCm) tensors used purely as device buffers; every step of the method runs inside the
library's HIP kernels. There is no CPU fallback: if the shared object is missing or the
tensors are not on the GPU the calls raise.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librsa.so")

RSA_RECTIFY_CRITICAL = 1
RSA_COMPENSATE = 2
RSA_DENSE = 4
RSA_MAX_BLOCKS = 4096
RSA_STATIC_SCRATCH_BYTES = 16 << 20
RSA_CACHE_CAUSAL = 1
RSA_CACHE_MAX_SELECT = 16384

EXPORTS = (
    "rsa_block_counts", "rsa_workspace_bytes", "rsa_pool", "rsa_pool_values", "rsa_implicit_attention", "rsa_adjacency_mask", "rsa_reorder_tokens", "rsa_select_blocks",
    "rsa_sparse_attn_rectified", "rsa_sparse_attn_rectified_static", "rsa_status_string",
    "rsa_cache_bytes", "rsa_cache_workspace_bytes", "rsa_cache_write", "rsa_cache_read", "rsa_cache_select", "rsa_cache_attn",
)


class RsaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = _lib().rsa_status_string(status).decode() if _LIB is not None else str(status)
        super().__init__(f"{where}: {msg} ({status})")


class rsa_shape(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("block", ctypes.c_int32),
        ("t_video", ctypes.c_int64), ("t_text", ctypes.c_int64),
        ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_t", ctypes.c_int64),
        ("scale", ctypes.c_float),
    ]


class rsa_cache(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("heads_kv", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("block", ctypes.c_int32),
        ("max_blocks", ctypes.c_int32), ("pages", ctypes.c_int64),
        ("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("k_mean", ctypes.c_void_p),
        ("table", ctypes.c_void_p),
    ]


class rsa_rows(ctypes.Structure):
    _fields_ = [
        ("heads", ctypes.c_int32), ("t", ctypes.c_int32),
        ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_t", ctypes.c_int64),
    ]


_LIB: Optional[ctypes.CDLL] = None


def _lib() -> ctypes.CDLL:
    """Load librsa.so (built by ``python -m paper_2511_19835_amd.build``); never falls back."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2511_19835_amd.build` "
                "(there is no fallback path)")
        lib = ctypes.CDLL(LIB_PATH)
        vp, i64p, szp = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_size_t)
        shp = ctypes.POINTER(rsa_shape)
        lib.rsa_block_counts.argtypes = [shp, i64p, i64p, i64p]
        lib.rsa_block_counts.restype = ctypes.c_int
        lib.rsa_workspace_bytes.argtypes = [shp, szp, szp]
        lib.rsa_workspace_bytes.restype = ctypes.c_int
        lib.rsa_pool.argtypes = [shp] + [vp] * 11 + [ctypes.c_int, vp, ctypes.c_size_t, vp]
        lib.rsa_pool.restype = ctypes.c_int
        lib.rsa_pool_values.argtypes = [shp, vp, vp, vp, vp]
        lib.rsa_pool_values.restype = ctypes.c_int
        lib.rsa_implicit_attention.argtypes = [shp] + [vp] * 7
        lib.rsa_implicit_attention.restype = ctypes.c_int
        lib.rsa_select_blocks.argtypes = [shp, vp, vp, ctypes.c_double, ctypes.c_double, vp, vp, vp, vp, vp, vp]
        lib.rsa_select_blocks.restype = ctypes.c_int
        lib.rsa_sparse_attn_rectified.argtypes = [shp] + [vp] * 10 + [ctypes.c_int, vp, vp, vp, ctypes.c_size_t, vp]
        lib.rsa_sparse_attn_rectified.restype = ctypes.c_int
        lib.rsa_sparse_attn_rectified_static.argtypes = [shp] + [vp] * 10 + [ctypes.c_int, vp, vp, vp]
        lib.rsa_sparse_attn_rectified_static.restype = ctypes.c_int
        lib.rsa_adjacency_mask.argtypes = [shp, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32), ctypes.c_int, vp, vp]
        lib.rsa_adjacency_mask.restype = ctypes.c_int
        lib.rsa_reorder_tokens.argtypes = [shp, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32), ctypes.c_int, vp, vp, vp]
        lib.rsa_reorder_tokens.restype = ctypes.c_int
        cap, rwp, i = ctypes.POINTER(rsa_cache), ctypes.POINTER(rsa_rows), ctypes.c_int
        lib.rsa_cache_bytes.argtypes = [cap, szp, szp, szp]
        lib.rsa_cache_bytes.restype = i
        lib.rsa_cache_workspace_bytes.argtypes = [cap, rwp, i, szp, szp]
        lib.rsa_cache_workspace_bytes.restype = i
        lib.rsa_cache_write.argtypes = [cap, rwp] + [vp] * 5
        lib.rsa_cache_write.restype = i
        lib.rsa_cache_read.argtypes = [cap, rwp] + [vp] * 5
        lib.rsa_cache_read.restype = i
        lib.rsa_cache_select.argtypes = [cap, rwp] + [vp] * 3 + [i] * 5 + [vp, vp, i, vp, ctypes.c_size_t, vp]
        lib.rsa_cache_select.restype = i
        lib.rsa_cache_attn.argtypes = [cap, rwp] + [vp] * 3 + [ctypes.c_float, i, vp, vp, i, i, vp, vp, vp, ctypes.c_size_t, vp]
        lib.rsa_cache_attn.restype = i
        lib.rsa_status_string.argtypes = [ctypes.c_int]
        lib.rsa_status_string.restype = ctypes.c_char_p
        _LIB = lib
    return _LIB


def load_library() -> ctypes.CDLL:
    return _lib()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise RsaError(status, where)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise RuntimeError("librsa takes device tensors only (no CPU path)")
    return t.data_ptr()


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def make_shape(q: torch.Tensor, t_video: int, t_text: int, block: int, scale: float = 0.0) -> rsa_shape:
    """Shape record for a [batch, heads, T, d] view of bf16 Q/K/V/O (any b/h/t strides)."""
    assert q.dim() == 4 and q.stride(3) == 1, "expect [batch, heads, tokens, head_dim], last dim contiguous"
    assert q.shape[2] == t_video + t_text
    return rsa_shape(q.shape[0], q.shape[1], q.shape[3], block, t_video, t_text,
                     q.stride(0), q.stride(1), q.stride(2), scale)


def rsa_block_counts(shape: rsa_shape):
    n, m, w = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    _check(_lib().rsa_block_counts(ctypes.byref(shape), ctypes.byref(n), ctypes.byref(m), ctypes.byref(w)),
           "rsa_block_counts")
    return n.value, m.value, w.value


def rsa_workspace_bytes(shape: rsa_shape):
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    _check(_lib().rsa_workspace_bytes(ctypes.byref(shape), ctypes.byref(a), ctypes.byref(b)), "rsa_workspace_bytes")
    return a.value, b.value


def rsa_pool(shape, Q, K, V, Qp, Kp, Vp, Vt, Spool, Apool, Lmass, Mc_bits, gapr_mode, ws, stream=None):
    _check(_lib().rsa_pool(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), _ptr(Qp), _ptr(Kp), _ptr(Vp), _ptr(Vt),
                           _ptr(Spool), _ptr(Apool), _ptr(Lmass), _ptr(Mc_bits), int(gapr_mode),
                           _ptr(ws), ws.numel() * ws.element_size() if ws is not None else 0,
                           _stream_ptr(stream)), "rsa_pool")


def rsa_implicit_attention(shape, K, Qp, Kp, Spool, Lmass, Apool, stream=None):
    _check(_lib().rsa_implicit_attention(ctypes.byref(shape), _ptr(K), _ptr(Qp), _ptr(Kp), _ptr(Spool), _ptr(Lmass),
                                         _ptr(Apool), _stream_ptr(stream)), "rsa_implicit_attention")


def rsa_pool_values(shape, V, Vp, Vt, stream=None):
    _check(_lib().rsa_pool_values(ctypes.byref(shape), _ptr(V), _ptr(Vp), _ptr(Vt), _stream_ptr(stream)),
           "rsa_pool_values")


def rsa_select_blocks(shape, Lmass, Apool, sparsity, p, forced_bits, mask_bits, block_idx, count, R, stream=None):
    _check(_lib().rsa_select_blocks(ctypes.byref(shape), _ptr(Lmass), _ptr(Apool), float(sparsity), float(p),
                                    _ptr(forced_bits), _ptr(mask_bits), _ptr(block_idx), _ptr(count), _ptr(R),
                                    _stream_ptr(stream)), "rsa_select_blocks")


def rsa_adjacency_mask(shape, grid, tile, radius, forced_bits, stream=None):
    g = (ctypes.c_int32 * 3)(*[int(x) for x in grid])
    t = (ctypes.c_int32 * 3)(*[int(x) for x in tile])
    _check(_lib().rsa_adjacency_mask(ctypes.byref(shape), g, t, int(radius), _ptr(forced_bits), _stream_ptr(stream)),
           "rsa_adjacency_mask")


def rsa_reorder_tokens(shape, grid, tile, direction, src, dst, stream=None):
    g = (ctypes.c_int32 * 3)(*[int(x) for x in grid])
    t = (ctypes.c_int32 * 3)(*[int(x) for x in tile])
    _check(_lib().rsa_reorder_tokens(ctypes.byref(shape), g, t, int(direction), _ptr(src), _ptr(dst),
                                     _stream_ptr(stream)), "rsa_reorder_tokens")


def rsa_sparse_attn_rectified(shape, Q, K, Vt, block_idx, count, mask_bits, R, Apool, Mc_bits, Vp, flags, O,
                              lse=None, ws=None, stream=None):
    _check(_lib().rsa_sparse_attn_rectified(
        ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(Vt), _ptr(block_idx), _ptr(count), _ptr(mask_bits), _ptr(R),
        _ptr(Apool), _ptr(Mc_bits), _ptr(Vp), int(flags), _ptr(O), _ptr(lse), _ptr(ws),
        ws.numel() * ws.element_size() if ws is not None else 0, _stream_ptr(stream)),
        "rsa_sparse_attn_rectified")


def rsa_sparse_attn_rectified_static(shape, Q, K, Vt, block_idx, count, mask_bits, R, Apool, Mc_bits, Vp, flags, O,
                                     lse=None, stream=None):
    _check(_lib().rsa_sparse_attn_rectified_static(
        ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(Vt), _ptr(block_idx), _ptr(count), _ptr(mask_bits), _ptr(R),
        _ptr(Apool), _ptr(Mc_bits), _ptr(Vp), int(flags), _ptr(O), _ptr(lse), _stream_ptr(stream)),
        "rsa_sparse_attn_rectified_static")


@dataclass
class LayerBuffers:
    """Caller-owned device buffers of one layer call, allocated once with torch."""
    shape: rsa_shape
    N: int
    M: int
    W: int
    Qp: torch.Tensor
    Kp: torch.Tensor
    Vp: torch.Tensor
    Vt: torch.Tensor
    Spool: torch.Tensor
    Apool: torch.Tensor
    Lmass: torch.Tensor
    Mc_bits: torch.Tensor
    mask_bits: torch.Tensor
    block_idx: torch.Tensor
    count: torch.Tensor
    R: torch.Tensor
    pool_ws: torch.Tensor
    attn_ws: Optional[torch.Tensor]


def allocate(q: torch.Tensor, t_video: int, t_text: int, block: int, scale: float = 0.0) -> LayerBuffers:
    shape = make_shape(q, t_video, t_text, block, scale)
    N, M, W = rsa_block_counts(shape)
    pool_ws, attn_ws = rsa_workspace_bytes(shape)
    B, H, _, d = q.shape
    dev = q.device
    f32 = dict(dtype=torch.float32, device=dev)
    i32 = dict(dtype=torch.int32, device=dev)
    return LayerBuffers(
        shape, N, M, W,
        Qp=torch.empty(B, H, N, d, **f32), Kp=torch.empty(B, H, M, d, **f32), Vp=torch.empty(B, H, M, d, **f32),
        Vt=torch.empty(B, H, M, d, block, dtype=torch.bfloat16, device=dev),
        Spool=torch.empty(B, H, N, M, **f32), Apool=torch.empty(B, H, N, M, **f32),
        Lmass=torch.empty(B, H, N, M, **f32),
        Mc_bits=torch.empty(B, H, N, W, **i32), mask_bits=torch.empty(B, H, N, W, **i32),
        block_idx=torch.empty(B, H, N, M, **i32), count=torch.empty(B, H, N, **i32), R=torch.empty(B, H, N, **f32),
        pool_ws=torch.empty(max(pool_ws, 256), dtype=torch.uint8, device=dev),
        attn_ws=torch.empty(attn_ws, dtype=torch.uint8, device=dev) if attn_ws else None,
    )


def rectified_sparse_attention(Q, K, V, O, buf: LayerBuffers, sparsity: float, p: float = 0.0,
                               gapr_mode: int = 1, forced_bits=None,
                               flags: int = RSA_RECTIFY_CRITICAL | RSA_COMPENSATE, lse=None, stream=None):
    """One layer: the three C-ABI calls back to back on one stream, no host sync."""
    rsa_pool(buf.shape, Q, K, V, buf.Qp, buf.Kp, buf.Vp, buf.Vt, buf.Spool, buf.Apool, buf.Lmass, buf.Mc_bits,
             gapr_mode, buf.pool_ws, stream)
    rsa_select_blocks(buf.shape, buf.Lmass, buf.Apool, sparsity, p, forced_bits, buf.mask_bits, buf.block_idx,
                      buf.count, buf.R, stream)
    rsa_sparse_attn_rectified(buf.shape, Q, K, buf.Vt, buf.block_idx, buf.count, buf.mask_bits, buf.R, buf.Apool,
                              buf.Mc_bits, buf.Vp, flags, O, lse, buf.attn_ws, stream)
    return O


# ---- the 8-bit key/value cache ---------------------------------------------------------
@dataclass
class KVCache:
    """Caller-owned device buffers of an 8-bit key/value cache and the record of them that the calls take."""
    desc: rsa_cache
    k_codes: torch.Tensor      # uint8 [pages, heads_kv, block * head_dim], opaque
    v_codes: torch.Tensor
    scales: torch.Tensor       # fp32  [pages, heads_kv, 4]
    k_mean: torch.Tensor       # int8  [pages, heads_kv, head_dim]
    table: torch.Tensor        # int32 [batch, max_blocks]: page of each block of a sequence, -1 where there is none

    def __post_init__(self):
        # what every call needs of the record, at hand
        self.ref = ctypes.byref(self.desc)
        self.device = self.k_codes.device
        self.batch, self.heads_kv, self.head_dim = self.desc.batch, self.desc.heads_kv, self.desc.head_dim


def cache_of(k_codes, v_codes, scales, k_mean, table, block: int) -> KVCache:
    """Record of a cache whose buffers exist. They may be filled and the table changed in place later."""
    pages, heads_kv, page = k_codes.shape
    want = ((k_codes, torch.uint8, (pages, heads_kv, page)), (v_codes, torch.uint8, (pages, heads_kv, page)),
            (scales, torch.float32, (pages, heads_kv, 4)), (k_mean, torch.int8, (pages, heads_kv, page // block)),
            (table, torch.int32, (table.shape[0], table.shape[-1])))
    for x, dtype, shape in want:
        if x.dtype != dtype or tuple(x.shape) != shape or not x.is_contiguous() or x.device != k_codes.device:
            raise ValueError(f"expect a contiguous {dtype} tensor of shape {shape} on {k_codes.device}, got {x.dtype} {tuple(x.shape)} on {x.device}")
    if page % block:
        raise ValueError(f"a page of {page} codes is no block of {block} tokens")
    desc = rsa_cache(table.shape[0], heads_kv, page // block, block, table.shape[1], pages, _ptr(k_codes), _ptr(v_codes),
                     _ptr(scales), _ptr(k_mean), _ptr(table))
    return KVCache(desc, k_codes, v_codes, scales, k_mean, table)


def allocate_cache(batch: int, heads_kv: int, head_dim: int, block: int, pages: int, max_blocks: int, device="cuda:0") -> KVCache:
    """An empty cache: no page is in the table yet."""
    probe = rsa_cache(batch, heads_kv, head_dim, block, max_blocks, pages)
    code, scale, mean = rsa_cache_bytes(probe)
    u8 = dict(dtype=torch.uint8, device=device)
    return cache_of(torch.empty(code, **u8).view(pages, heads_kv, block * head_dim),
                    torch.empty(code, **u8).view(pages, heads_kv, block * head_dim),
                    torch.empty(scale // 4, dtype=torch.float32, device=device).view(pages, heads_kv, 4),
                    torch.empty(mean, dtype=torch.int8, device=device).view(pages, heads_kv, head_dim),
                    torch.full((batch, max_blocks), -1, dtype=torch.int32, device=device), block)


def make_rows(x: torch.Tensor) -> rsa_rows:
    """Row record of a [batch, heads, t, head_dim] bf16 view (any b/h/t strides): new keys and values, or queries and outputs."""
    assert x.dim() == 4 and x.stride(3) == 1 and x.dtype == torch.bfloat16, "expect bf16 [batch, heads, t, head_dim], last dim contiguous"
    # (torch leaves the stride of a dimension of one element open)
    sb, sh, st = (x.stride(i) if x.shape[i] > 1 else -(-x.shape[3] // 8) * 8 for i in range(3))
    rows = rsa_rows(x.shape[1], x.shape[2], sb, sh, st)
    rows.shape, rows.strides, rows.ref = x.shape, x.stride(), ctypes.byref(rows)
    return rows


def _row_tensor(cache: KVCache, rows: rsa_rows, x: torch.Tensor) -> int:
    """Address of a tensor that goes with a row record: bf16, of its sizes and strides, on the cache's device."""
    shape = x.shape
    if (x.dtype is not torch.bfloat16 or shape != rows.shape or shape[0] != cache.batch or shape[3] != cache.head_dim or x.device != cache.device
            or x.stride() != rows.strides and any(n > 1 and p != q for n, p, q in zip(shape, x.stride(), rows.strides))):
        raise ValueError(f"tensor {x.dtype} {tuple(shape)} strides {x.stride()} on {x.device} is not what the row record says")
    return x.data_ptr()


def _lengths(cache: KVCache, x: Optional[torch.Tensor]) -> Optional[int]:
    if x is None:
        return None
    if x.dtype is not torch.int32 or x.numel() != cache.batch or not x.is_contiguous() or x.device != cache.device:
        raise ValueError("expect contiguous int32 lengths, one for each sequence, on the cache's device")
    return x.data_ptr()


def _lists(cache: KVCache, rows: rsa_rows, group: int, block_idx: torch.Tensor, kept: torch.Tensor) -> None:
    shape = (cache.batch, cache.heads_kv, -(-rows.shape[2] // max(1, group)))
    if (block_idx.dtype is not torch.int32 or kept.dtype is not torch.int32 or block_idx.dim() != 4 or block_idx.shape[:3] != shape or kept.shape != shape
            or not block_idx.is_contiguous() or not kept.is_contiguous() or block_idx.device != cache.device or kept.device != cache.device):
        raise ValueError(f"expect contiguous int32 lists {shape} + [list_len] and counts {shape} on the cache's device")


def _call(cache: KVCache, stream, where: str, fn, *args) -> None:
    """One call on the cache's device: on `stream`, or on that device's current stream."""
    dev = cache.device.index
    raw = torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream
    if torch.cuda.current_device() == dev:
        status = fn(cache.ref, *args, raw)
    else:
        with torch.cuda.device(dev):
            status = fn(cache.ref, *args, raw)
    if status != 0:
        raise RsaError(status, where)


def _scratch(cache: KVCache, ws: Optional[torch.Tensor]):
    if ws is None:
        return None, 0
    if not ws.is_contiguous() or ws.device != cache.device:
        raise ValueError(f"expect a contiguous workspace on {cache.device}, got strides {ws.stride()} on {ws.device}")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def rsa_cache_bytes(desc: rsa_cache):
    a, b, c = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check(_lib().rsa_cache_bytes(ctypes.byref(desc), ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)), "rsa_cache_bytes")
    return a.value, b.value, c.value


def rsa_cache_workspace_bytes(cache: KVCache, rows: rsa_rows, group: int = 0):
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    _check(_lib().rsa_cache_workspace_bytes(cache.ref, rows.ref, int(group), ctypes.byref(a), ctypes.byref(b)),
           "rsa_cache_workspace_bytes")
    return a.value, b.value


def rsa_cache_write(cache: KVCache, rows, K, V, start, count=None, stream=None):
    _call(cache, stream, "rsa_cache_write", _lib().rsa_cache_write, rows.ref, _row_tensor(cache, rows, K), _row_tensor(cache, rows, V),
          _lengths(cache, start), _lengths(cache, count))


def rsa_cache_read(cache: KVCache, rows, start, count, K, V, stream=None):
    _call(cache, stream, "rsa_cache_read", _lib().rsa_cache_read, rows.ref, _lengths(cache, start), _lengths(cache, count),
          _row_tensor(cache, rows, K), _row_tensor(cache, rows, V))


def rsa_cache_select(cache: KVCache, rows, Q, kv_len, q_len, group, keep, first, last, flags, block_idx, kept, ws=None, stream=None):
    _lists(cache, rows, group, block_idx, kept)
    _call(cache, stream, "rsa_cache_select", _lib().rsa_cache_select, rows.ref, _row_tensor(cache, rows, Q), _lengths(cache, kv_len),
          _lengths(cache, q_len), group, keep, first, last, flags, block_idx.data_ptr(), kept.data_ptr(), block_idx.shape[3], *_scratch(cache, ws))


def rsa_cache_attn(cache: KVCache, rows, Q, kv_len, q_len, scale, flags, block_idx, kept, group, O, lse=None, ws=None, stream=None):
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != rows.shape[:3] or not lse.is_contiguous() or lse.device != cache.device):
        raise ValueError("expect a contiguous fp32 lse [batch, heads, t] on the cache's device")
    if block_idx is not None and kept is not None:
        _lists(cache, rows, group, block_idx, kept)
    _call(cache, stream, "rsa_cache_attn", _lib().rsa_cache_attn, rows.ref, _row_tensor(cache, rows, Q), _lengths(cache, kv_len),
          _lengths(cache, q_len), scale, flags, _ptr(block_idx), _ptr(kept), group, block_idx.shape[3] if block_idx is not None else 0,
          _row_tensor(cache, rows, O), _ptr(lse), *_scratch(cache, ws))


def cached_sparse_attention(cache: KVCache, K, V, Q, O, kv_len, q_len, group: int, keep: int, block_idx, kept, first: int = 1,
                            last: int = 1, flags: int = RSA_CACHE_CAUSAL, start=None, lse=None, ws=None, stream=None):
    """One step of a sequence of frames or tokens: the new rows into the cache, the blocks that each group of them reads, and
    their attention; three C-ABI calls on one stream, no host sync. `kv_len` counts the new rows, `start` = kv_len - q_len
    (computed here when it is not given; a q_len of more than all rows counts as all). `ws` holds the larger of the two
    workspaces: the calls use it one after the other."""
    if K.shape[2] != Q.shape[2]:
        raise ValueError(f"a step brings keys and queries for the same rows: got {K.shape[2]} and {Q.shape[2]}")
    if start is None:
        with torch.cuda.stream(stream):                # (None: the current stream)
            start = kv_len - (q_len.clamp(max=Q.shape[2]) if q_len is not None else Q.shape[2])
    rows_kv, rows = make_rows(K), make_rows(Q)
    rsa_cache_write(cache, rows_kv, K, V, start, q_len, stream)
    rsa_cache_select(cache, rows, Q, kv_len, q_len, group, keep, first, last, flags, block_idx, kept, ws, stream)
    rsa_cache_attn(cache, rows, Q, kv_len, q_len, 0.0, flags, block_idx, kept, group, O, lse, ws, stream)
    return O
