"""Thin ctypes binding of librsa.so: argument marshalling only.

The entry points carry the names of the C-ABI (include/rsa.h). Tensors are torch CUDA
(ROCm) tensors used purely as device buffers; every step of the method runs inside the
library's HIP kernels. There is no CPU fallback: if the shared object is missing or the
tensors are not on the GPU the calls raise.
"""
from __future__ import annotations

import ctypes
import math
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
RSA_ROTARY_PLAIN, RSA_ROTARY_LINEAR, RSA_ROTARY_BASE, RSA_ROTARY_PARTS = 0, 1, 2, 3
RSA_ROTARY_INVERSE = 1

EXPORTS = (
    "rsa_block_counts", "rsa_workspace_bytes", "rsa_pool", "rsa_pool_values", "rsa_implicit_attention", "rsa_adjacency_mask", "rsa_reorder_tokens", "rsa_select_blocks",
    "rsa_sparse_attn_rectified", "rsa_sparse_attn_rectified_static", "rsa_status_string",
    "rsa_cache_bytes", "rsa_cache_workspace_bytes", "rsa_cache_write", "rsa_cache_read", "rsa_cache_select", "rsa_cache_attn",
    "rsa_fourbit_bytes", "rsa_fourbit_workspace_bytes", "rsa_fourbit_write", "rsa_fourbit_read", "rsa_fourbit_attn",
    "rsa_cache_assign", "rsa_rotary_frequencies", "rsa_rotary_apply",
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


class rsa_pages(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("max_blocks", ctypes.c_int32), ("block", ctypes.c_int32), ("pages", ctypes.c_int64),
        ("table", ctypes.c_void_p), ("free_pages", ctypes.c_void_p),
    ]


class rsa_rotary(ctypes.Structure):
    _fields_ = [
        ("head_dim", ctypes.c_int32), ("pairs", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("axes", ctypes.c_int32),
        ("axis_pairs", ctypes.c_int32 * 3), ("factor", ctypes.c_float), ("freq", ctypes.c_void_p),
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
        lib.rsa_fourbit_bytes.argtypes = [cap, szp, szp, szp, szp]
        lib.rsa_fourbit_workspace_bytes.argtypes = [cap, rwp, i, szp]
        lib.rsa_fourbit_write.argtypes = lib.rsa_cache_write.argtypes
        lib.rsa_fourbit_read.argtypes = lib.rsa_cache_read.argtypes
        lib.rsa_fourbit_attn.argtypes = lib.rsa_cache_attn.argtypes
        lib.rsa_cache_assign.argtypes = [ctypes.POINTER(rsa_pages), i] + [vp] * 11
        dbl = ctypes.c_double
        lib.rsa_rotary_frequencies.argtypes = [i, dbl, i, dbl, dbl, dbl, dbl, ctypes.POINTER(dbl), ctypes.POINTER(ctypes.c_float)]
        lib.rsa_rotary_apply.argtypes = [ctypes.POINTER(rsa_rotary), i, rwp, vp, vp, rwp, vp, vp, vp, vp, vp, i, vp]
        for name in EXPORTS[17:]:
            getattr(lib, name).restype = i
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


# ---- the key/value cache in 8 and in 4 bits ----------------------------------------------
@dataclass
class KVCache:
    """Caller-owned device buffers of a key/value cache and the record of them that the calls take."""
    desc: rsa_cache
    k_codes: torch.Tensor      # uint8 [pages, heads_kv, block * head_dim], opaque (4 bits: block * (head_dim / 2 + head_dim / 32))
    v_codes: torch.Tensor      # the same (4 bits: block * (head_dim / 2 + 2))
    scales: torch.Tensor       # fp32  [pages, heads_kv, 4]
    k_mean: torch.Tensor       # int8  [pages, heads_kv, head_dim]
    table: torch.Tensor        # int32 [batch, max_blocks]: page of each block of a sequence, -1 where there is none
    bits: int = 8

    def __post_init__(self):
        # what every call needs of the record, at hand
        self.ref = ctypes.byref(self.desc)
        self.device = self.k_codes.device
        self.dev = self.device.index
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


def fourbit_of(k_codes, v_codes, scales, k_mean, table, block: int) -> KVCache:
    """Record of a cache in 4 bits whose buffers exist."""
    pages, heads_kv, head_dim = k_mean.shape
    want = ((k_codes, torch.uint8, (pages, heads_kv, block * (head_dim // 2 + head_dim // 32))),
            (v_codes, torch.uint8, (pages, heads_kv, block * (head_dim // 2 + 2))), (scales, torch.float32, (pages, heads_kv, 4)),
            (k_mean, torch.int8, (pages, heads_kv, head_dim)), (table, torch.int32, (table.shape[0], table.shape[-1])))
    for x, dtype, shape in want:
        if x.dtype != dtype or tuple(x.shape) != shape or not x.is_contiguous() or x.device != k_codes.device:
            raise ValueError(f"expect a contiguous {dtype} tensor of shape {shape} on {k_codes.device}, got {x.dtype} {tuple(x.shape)} on {x.device}")
    desc = rsa_cache(table.shape[0], heads_kv, head_dim, block, table.shape[1], pages, _ptr(k_codes), _ptr(v_codes), _ptr(scales),
                     _ptr(k_mean), _ptr(table))
    return KVCache(desc, k_codes, v_codes, scales, k_mean, table, 4)


def allocate_cache(batch: int, heads_kv: int, head_dim: int, block: int, pages: int, max_blocks: int, device="cuda:0", bits: int = 8) -> KVCache:
    """An empty cache of 8 or 4 bits: no page is in the table yet."""
    if bits not in (4, 8):
        raise ValueError(f"a cache holds 8 or 4 bits, not {bits}")
    probe = rsa_cache(batch, heads_kv, head_dim, block, max_blocks, pages)
    if bits == 4:
        sizes = rsa_fourbit_bytes(probe)
        k, v = (torch.empty(n, dtype=torch.uint8, device=device).view(pages, heads_kv, -1) for n in sizes[:2])
        return fourbit_of(k, v, torch.empty(pages, heads_kv, 4, dtype=torch.float32, device=device),
                          torch.empty(pages, heads_kv, head_dim, dtype=torch.int8, device=device),
                          torch.full((batch, max_blocks), -1, dtype=torch.int32, device=device), block)
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


# (The checks of a call cost more than its launch where it is small: each asks a tensor as little as will do.)
_I32, _I64, _BF16 = torch.int32, torch.int64, torch.bfloat16


def _row_addresses(cache, rows: rsa_rows, *xs) -> list:
    """Addresses of tensors that go with a row record: bf16, of its sizes and strides, on the device of the cache (or of the frequencies)."""
    shape, strides, dev = rows.shape, rows.strides, cache.dev
    out = []
    for x in xs:
        if (x.dtype is not _BF16 or x.shape != shape or x.get_device() != dev
                or x.stride() != strides and any(n > 1 and p != q for n, p, q in zip(shape, x.stride(), strides))):
            raise ValueError(f"tensor {x.dtype} {tuple(x.shape)} strides {x.stride()} on {x.device} is not what the row record says")
        out.append(x.data_ptr())
    return out


def _cache_rows(cache: KVCache, rows: rsa_rows, *xs) -> list:
    if rows.shape[0] != cache.batch or rows.shape[3] != cache.head_dim:
        raise ValueError(f"rows {tuple(rows.shape)} are not those of {cache.batch} sequences with heads of {cache.head_dim}")
    return _row_addresses(cache, rows, *xs)


def _vectors(dev: int, n: int, *xs) -> list:
    """Addresses of contiguous int32 tensors of n elements on device `dev`; None for None."""
    out = []
    for x in xs:
        if x is None:
            out.append(None)
            continue
        if x.dtype is not _I32 or x.numel() != n or x.get_device() != dev or not x.is_contiguous():
            raise ValueError(f"expect {n} contiguous int32 numbers on cuda:{dev}, got {x.dtype} {tuple(x.shape)} on {x.device}")
        out.append(x.data_ptr())
    return out


def _lists(cache: KVCache, rows: rsa_rows, group: int, block_idx: torch.Tensor, kept: torch.Tensor) -> None:
    shape = (cache.batch, cache.heads_kv, -(-rows.shape[2] // max(1, group)))
    if (block_idx.dtype is not torch.int32 or kept.dtype is not torch.int32 or block_idx.dim() != 4 or block_idx.shape[:3] != shape or kept.shape != shape
            or not block_idx.is_contiguous() or not kept.is_contiguous() or block_idx.device != cache.device or kept.device != cache.device):
        raise ValueError(f"expect contiguous int32 lists {shape} + [list_len] and counts {shape} on the cache's device")


def _launch(dev: int, stream, where: str, fn, *args) -> None:
    """One call on a device: on `stream`, or on that device's current stream."""
    raw = torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream
    if torch._C._cuda_getDevice() == dev:
        status = fn(*args, raw)
    else:
        with torch.cuda.device(dev):
            status = fn(*args, raw)
    if status != 0:
        raise RsaError(status, where)


def _of_bits(cache: KVCache, bits: int, where: str) -> None:
    if cache.bits != bits:
        raise ValueError(f"{where} takes a cache of {bits} bits, not of {cache.bits}")


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
    _of_bits(cache, 8, "rsa_cache_write")
    _launch(cache.dev, stream, "rsa_cache_write", _lib().rsa_cache_write, cache.ref, rows.ref, *_cache_rows(cache, rows, K, V),
            *_vectors(cache.dev, cache.batch, start, count))


def rsa_cache_read(cache: KVCache, rows, start, count, K, V, stream=None):
    _of_bits(cache, 8, "rsa_cache_read")
    _launch(cache.dev, stream, "rsa_cache_read", _lib().rsa_cache_read, cache.ref, rows.ref, *_vectors(cache.dev, cache.batch, start, count),
            *_cache_rows(cache, rows, K, V))


def rsa_cache_select(cache: KVCache, rows, Q, kv_len, q_len, group, keep, first, last, flags, block_idx, kept, ws=None, stream=None):
    _lists(cache, rows, group, block_idx, kept)
    _launch(cache.dev, stream, "rsa_cache_select", _lib().rsa_cache_select, cache.ref, rows.ref, *_cache_rows(cache, rows, Q),
            *_vectors(cache.dev, cache.batch, kv_len, q_len), group, keep, first, last, flags, block_idx.data_ptr(), kept.data_ptr(),
            block_idx.shape[3], *_scratch(cache, ws))


def _attn_call(cache: KVCache, where: str, fn, bits: int, rows, Q, kv_len, q_len, scale, flags, block_idx, kept, group, O, lse, ws, stream):
    _of_bits(cache, bits, where)
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != rows.shape[:3] or lse.get_device() != cache.dev or not lse.is_contiguous()):
        raise ValueError("expect a contiguous fp32 lse [batch, heads, t] on the cache's device")
    if block_idx is not None and kept is not None:
        _lists(cache, rows, group, block_idx, kept)
    q, o = _cache_rows(cache, rows, Q, O)
    _launch(cache.dev, stream, where, fn, cache.ref, rows.ref, q, *_vectors(cache.dev, cache.batch, kv_len, q_len), scale, flags, _ptr(block_idx),
            _ptr(kept), group, block_idx.shape[3] if block_idx is not None else 0, o, lse.data_ptr() if lse is not None else None, *_scratch(cache, ws))


def rsa_cache_attn(cache: KVCache, rows, Q, kv_len, q_len, scale, flags, block_idx, kept, group, O, lse=None, ws=None, stream=None):
    _attn_call(cache, "rsa_cache_attn", _lib().rsa_cache_attn, 8, rows, Q, kv_len, q_len, scale, flags, block_idx, kept, group, O, lse, ws, stream)


def rsa_fourbit_bytes(desc: rsa_cache):
    out = [ctypes.c_size_t() for _ in range(4)]
    _check(_lib().rsa_fourbit_bytes(ctypes.byref(desc), *(ctypes.byref(x) for x in out)), "rsa_fourbit_bytes")
    return tuple(x.value for x in out)


def rsa_fourbit_workspace_bytes(cache: KVCache, rows: rsa_rows, group: int = 0):
    a = ctypes.c_size_t()
    _check(_lib().rsa_fourbit_workspace_bytes(cache.ref, rows.ref, int(group), ctypes.byref(a)), "rsa_fourbit_workspace_bytes")
    return a.value


def rsa_fourbit_write(cache: KVCache, rows, K, V, start, count=None, stream=None):
    _of_bits(cache, 4, "rsa_fourbit_write")
    _launch(cache.dev, stream, "rsa_fourbit_write", _lib().rsa_fourbit_write, cache.ref, rows.ref, *_cache_rows(cache, rows, K, V),
            *_vectors(cache.dev, cache.batch, start, count))


def rsa_fourbit_read(cache: KVCache, rows, start, count, K, V, stream=None):
    _of_bits(cache, 4, "rsa_fourbit_read")
    _launch(cache.dev, stream, "rsa_fourbit_read", _lib().rsa_fourbit_read, cache.ref, rows.ref, *_vectors(cache.dev, cache.batch, start, count),
            *_cache_rows(cache, rows, K, V))


def rsa_fourbit_attn(cache: KVCache, rows, Q, kv_len, q_len, scale, flags, block_idx, kept, group, O, lse=None, ws=None, stream=None):
    _attn_call(cache, "rsa_fourbit_attn", _lib().rsa_fourbit_attn, 4, rows, Q, kv_len, q_len, scale, flags, block_idx, kept, group, O, lse, ws, stream)


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
    write, attn = (rsa_fourbit_write, rsa_fourbit_attn) if cache.bits == 4 else (rsa_cache_write, rsa_cache_attn)
    write(cache, rows_kv, K, V, start, q_len, stream)
    rsa_cache_select(cache, rows, Q, kv_len, q_len, group, keep, first, last, flags, block_idx, kept, ws, stream)
    attn(cache, rows, Q, kv_len, q_len, 0.0, flags, block_idx, kept, group, O, lse, ws, stream)
    return O


# ---- pages, positions and a step of many requests ----------------------------------------
@dataclass
class Pages:
    """A cache's table and the list of pages that no sequence holds, and the record of them."""
    desc: rsa_pages
    table: torch.Tensor        # int32 [batch, max_blocks]
    free_pages: torch.Tensor   # int32 [pages]

    def __post_init__(self):
        self.ref, self.device, self.dev, self.batch = ctypes.byref(self.desc), self.table.device, self.table.device.index, self.desc.batch


def pages_of(table: torch.Tensor, free_pages: torch.Tensor, block: int) -> Pages:
    """Record of a table and a free list; free_pages has room for every page of the cache."""
    for x, dims in ((table, 2), (free_pages, 1)):
        if x.dtype is not torch.int32 or x.dim() != dims or not x.is_contiguous() or x.device != table.device:
            raise ValueError(f"expect a contiguous int32 tensor of {dims} dimensions on {table.device}, got {x.dtype} {tuple(x.shape)} on {x.device}")
    return Pages(rsa_pages(table.shape[0], table.shape[1], block, free_pages.shape[0], _ptr(table), _ptr(free_pages)), table, free_pages)


def rsa_cache_assign(pages: Pages, t, kv_len, add, free_count, kv_new, free_left, start, count, positions=None, slots=None, shared=None, stream=None):
    n, dev = pages.batch, pages.dev
    kv, more, own, new, first, many = _vectors(dev, n, kv_len, add, shared, kv_new, start, count)
    free, left = _vectors(dev, 1, free_count, free_left)
    pos, = _vectors(dev, n * t, positions)
    slot = None
    if slots is not None:
        if slots.dtype is not _I64 or slots.numel() != n * t or slots.get_device() != dev or not slots.is_contiguous():
            raise ValueError(f"expect {n * t} contiguous int64 slots on cuda:{dev}, got {slots.dtype} {tuple(slots.shape)} on {slots.device}")
        slot = slots.data_ptr()
    _launch(dev, stream, "rsa_cache_assign", _lib().rsa_cache_assign, pages.ref, t, kv, more, own, free, new, left, first, many, pos, slot)


@dataclass
class Rotary:
    """Frequencies of rotary positions on the device and the record of them."""
    desc: rsa_rotary
    freq: torch.Tensor         # fp64 [pairs], radians a position

    def __post_init__(self):
        # (what rsa_rotary_apply refuses of the record, before a step has moved anything on; the factor as fp32 holds it)
        if self.desc.pairs < 1 or not 0 <= self.desc.factor < math.inf:
            raise ValueError(f"expect at least one pair and a finite factor of at least 0: got {self.desc.pairs} and {self.desc.factor}")
        self.device, self.dev, self.axes, self.refs = self.freq.device, self.freq.device.index, self.desc.axes, {}

    def ref(self, head_dim: int):
        """The record for heads of `head_dim` channels."""
        if head_dim not in self.refs:          # (one for each size of heads)
            d = rsa_rotary.from_buffer_copy(self.desc)
            d.head_dim = head_dim
            self.refs[head_dim] = ctypes.byref(d)
        return self.refs[head_dim]


def make_rotary(freq: torch.Tensor, pairing: str = "half", axis_pairs=None, factor: float = 1.0) -> Rotary:
    """Record of fp64 frequencies on the device, one for each pair of channels that turns. pairing: "half" (channels j and pairs + j) or
    "interleaved" (2 j and 2 j + 1); axis_pairs: how many of the pairs turn along each of up to three axes."""
    if pairing not in ("half", "interleaved"):
        raise ValueError(f"pairs are 'half' or 'interleaved', not {pairing!r}")
    if freq.dtype is not torch.float64 or freq.dim() != 1 or not freq.is_contiguous():
        raise ValueError(f"expect contiguous fp64 frequencies of one dimension, got {freq.dtype} {tuple(freq.shape)}")
    axis = list(axis_pairs) if axis_pairs is not None else [freq.shape[0]]
    if not 1 <= len(axis) <= 3 or sum(axis) != freq.shape[0] or min(axis) < 0:
        raise ValueError(f"pairs of up to three axes add up to {freq.shape[0]}: got {axis}")
    rot = Rotary(rsa_rotary(0, freq.shape[0], int(pairing == "interleaved"), len(axis), (ctypes.c_int32 * 3)(*axis), float(factor), None), freq)
    rot.desc.freq = _ptr(freq)
    return rot


def rsa_rotary_frequencies(pairs: int, base: float = 10000.0, scaling: int = RSA_ROTARY_PLAIN, stretch: float = 1.0, old_len: float = 0.0,
                           turns_few: float = 1.0, turns_many: float = 32.0):
    """(frequencies as a list, factor) of one axis."""
    freq, factor = (ctypes.c_double * max(1, pairs))(), ctypes.c_float()
    _check(_lib().rsa_rotary_frequencies(pairs, base, scaling, stretch, old_len, turns_few, turns_many, freq, ctypes.byref(factor)), "rsa_rotary_frequencies")
    return list(freq), factor.value


def rsa_rotary_apply(rotary: Rotary, rows_q, Q, Qr, rows_k=None, K=None, Kr=None, positions=None, start=None, count=None, flags=0, stream=None):
    b, _, t, d = rows_q.shape
    dev = rotary.dev
    q, qr = _row_addresses(rotary, rows_q, Q, Qr)
    ref = k = kr = None
    if rows_k is not None:
        if rows_k.shape[0] != b or rows_k.shape[3] != d:
            raise ValueError(f"queries and keys are of the same sequences and head sizes: got {tuple(rows_q.shape)} and {tuple(rows_k.shape)}")
        ref, (k, kr) = rows_k.ref, _row_addresses(rotary, rows_k, K, Kr)
    if positions is not None and tuple(positions.shape) != (rotary.axes, b, t) and (rotary.axes, *positions.shape) != (1, b, t):
        raise ValueError(f"expect positions {(rotary.axes, b, t)}, got {tuple(positions.shape)}")
    pos, = _vectors(dev, rotary.axes * b * t, positions)
    first, many = _vectors(dev, b, start, count)
    _launch(dev, stream, "rsa_rotary_apply", _lib().rsa_rotary_apply, rotary.ref(d), b, rows_q.ref, q, qr, ref, k, kr, pos, first, many, flags)


def serve_step(cache: KVCache, pages: Pages, rotary: Rotary, Q, K, V, O, kv_len, add, free_count, start, count, positions=None, slots=None, shared=None,
               lse=None, ws=None, stream=None):
    """One step of a batch of requests on one stream, with no host sync, so that it can be captured and replayed: sequence b brings add[b] new
    tokens (rows 0 .. add[b] - 1 of Q, K and V; less than 0: it is cut). Pages for them (rsa_cache_assign; kv_len, free_count and shared move on in place,
    start and count say what was served), Q and K turned in place by their positions, keys and values into the cache, and the causal
    attention of the new queries over their sequences. Rows of sequences that were not served are left as they were. Q, K and V must not overlap.
    ws: bytes of the attention's workspace (rsa_fourbit_workspace_bytes, or the second of rsa_cache_workspace_bytes); None: the keys of a tile are not
    split over workgroups, which takes many times as long for few new tokens of few long sequences. Positions are along one axis and the attention
    is over all blocks: other steps are put together of the same four calls."""
    # (all of it before the first call: that one moves the lengths on)
    if (pages.table.data_ptr() != cache.table.data_ptr() or pages.desc.block != cache.desc.block or pages.batch != cache.batch
            or pages.desc.pages != cache.desc.pages):
        raise ValueError("the pages are not those of the cache's table")
    if K.shape[2] != Q.shape[2] or rotary.dev != cache.dev:
        raise ValueError(f"a step brings keys and queries for the same rows, on one device: got {K.shape[2]} and {Q.shape[2]} rows")
    rows, rows_kv = make_rows(Q), make_rows(K)
    _cache_rows(cache, rows, Q, O)
    _cache_rows(cache, rows_kv, K, V)
    if K.shape[1] != cache.heads_kv or Q.shape[1] % cache.heads_kv or 2 * rotary.desc.pairs > cache.head_dim:
        raise ValueError(f"{Q.shape[1]} and {K.shape[1]} heads of {cache.head_dim} channels, {rotary.desc.pairs} pairs: not for a cache of {cache.heads_kv} heads")
    if rotary.axes != 1:
        raise ValueError("a step's tokens stand in a row: positions along one axis")
    if Q.shape[0] * Q.shape[2] * (cache.head_dim // 8 + 2) // 64 >= 1 << 23 or Q.shape[1] + K.shape[1] > 65535:
        raise ValueError(f"{Q.shape[0]} times {Q.shape[2]} rows of {Q.shape[1]} and {K.shape[1]} heads are more than rsa_rotary_apply takes")
    write, attn = (rsa_fourbit_write, rsa_fourbit_attn) if cache.bits == 4 else (rsa_cache_write, rsa_cache_attn)
    at = [x.data_ptr() for x in (Q, K, V, O)]
    if any(x % 16 for x in at) or at[0] == at[1] or at[2] in at[:2]:
        raise ValueError("queries, keys, values and outputs begin at multiples of 16 bytes, and queries, keys and values are three tensors")
    sizes = rsa_fourbit_workspace_bytes if cache.bits == 4 else lambda *x: rsa_cache_workspace_bytes(*x)[1]
    need, _ = sizes(cache, rows), sizes(cache, rows_kv)          # (strides that the calls do not take raise here)
    if ws is not None:
        where, size = _scratch(cache, ws)
        if size < need or where % 256:
            raise ValueError(f"the attention's workspace has {need} bytes, from a multiple of 256 on")
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != rows.shape[:3] or lse.get_device() != cache.dev or not lse.is_contiguous()):
        raise ValueError("expect a contiguous fp32 lse [batch, heads, t] on the cache's device")
    rsa_cache_assign(pages, Q.shape[2], kv_len, add, free_count, kv_len, free_count, start, count, positions, slots, shared, stream)
    rsa_rotary_apply(rotary, rows, Q, Q, rows_kv, K, K, None, start, count, 0, stream)
    write(cache, rows_kv, K, V, start, count, stream)
    attn(cache, rows, Q, kv_len, count, 0.0, RSA_CACHE_CAUSAL, None, None, 0, O, lse, ws, stream)
    return O
