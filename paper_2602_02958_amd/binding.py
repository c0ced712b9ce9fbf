"""Thin ctypes binding of libqvg.so (include/qvg.h): argument marshalling only.

Every step of the codec runs in the library's HIP kernels; this module converts torch
tensors to device pointers, allocates outputs and workspace with torch, passes torch's
current stream, and raises on a negative status.  It never falls back to a CPU path:
a missing library raises at the first call.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import os
from array import array
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libqvg.so")
_lib = None

ENTRY_ENCODE, ENTRY_DECODE, ENTRY_ATTN, ENTRY_KMEANS_UPDATE, ENTRY_KMEANS_ASSIGN = 0, 1, 2, 3, 4
SCALE_F16, SCALE_E4M3 = 0, 1
TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}      # QVG_BF16, QVG_F16, QVG_F32

EXPORTS = ["qvg_encode_chunk", "qvg_encode_chunk_static", "qvg_decode", "qvg_decode_ex", "qvg_attn_decode", "qvg_attn_decode_ex",
           "qvg_attn_decode_causal", "qvg_attn_decode_f32", "qvg_attn_decode_parts", "qvg_attn_scratch_bytes", "qvg_attn_scratch_bytes_causal",
           "qvg_attn_merge",
           "qvg_attn_tree", "qvg_attn_tree_scratch_bytes", "qvg_tree_mask", "qvg_keep_nodes", "qvg_copy_pages",
           "qvg_rope_table", "qvg_rope", "qvg_append_pages", "qvg_attn_pages", "qvg_attn_pages_scratch_bytes",
           "qvg_kmeans_assign",
           "qvg_kmeans_update", "qvg_workspace_bytes", "qvg_compressed_bytes",
           "qvg_status_string", "qvg_version"]


class QvgParams(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("head_dim", C.c_int32), ("n_clusters", C.c_int32),
                ("group_size", C.c_int32), ("n_stages", C.c_int32), ("bits", C.c_int32),
                ("n_smooth_stages", C.c_int32), ("kmeans_iters", C.c_int32), ("scale_format", C.c_int32)]


class QvgTreeStep(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("group", C.c_int32), ("n_nodes", C.c_int32), ("table_pages", C.c_int32),
                ("page_len", C.c_int64), ("pool_pages", C.c_int64), ("page_table", C.c_void_p), ("kv_len", C.c_void_p),
                ("q", C.c_void_p), ("q_stride_seq", C.c_int64), ("q_stride_head", C.c_int64), ("q_stride_node", C.c_int64),
                ("k_new", C.c_void_p), ("v_new", C.c_void_p),
                ("new_stride_seq", C.c_int64), ("new_stride_head", C.c_int64), ("new_stride_node", C.c_int64),
                ("k_tail", C.c_void_p), ("v_tail", C.c_void_p),
                ("tail_stride_seq", C.c_int64), ("tail_stride_head", C.c_int64), ("tail_stride_token", C.c_int64),
                ("tail_len", C.c_void_p), ("tail_capacity", C.c_int32), ("reserved", C.c_int32),
                ("nodes", C.c_void_p), ("mask", C.c_void_p), ("k_rope_f16", C.c_void_p), ("rope_tokens", C.c_int64),
                ("out", C.c_void_p), ("out_stride_seq", C.c_int64), ("out_stride_head", C.c_int64), ("out_stride_node", C.c_int64),
                ("lse", C.c_void_p)]


class QvgRotary(C.Structure):
    _fields_ = [("table", C.c_void_p), ("type", C.c_int32), ("n_pairs", C.c_int32), ("n_rows", C.c_int64), ("half", C.c_int32),
                ("reserved", C.c_int32), ("positions", C.c_void_p)]


class QvgPageCache(C.Structure):
    _fields_ = [("type", C.c_int32), ("n_seqs", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32), ("table_pages", C.c_int32),
                ("reserved", C.c_int32), ("page_len", C.c_int64), ("pool_pages", C.c_int64), ("page_table", C.c_void_p), ("kv_len", C.c_void_p),
                ("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("stride_head", C.c_int64), ("stride_page", C.c_int64),
                ("stride_token", C.c_int64)]


class QvgPageStep(C.Structure):
    _fields_ = [("group", C.c_int32), ("n_new", C.c_int32), ("n_live", C.c_void_p), ("q", C.c_void_p), ("q_stride_seq", C.c_int64),
                ("q_stride_head", C.c_int64), ("q_stride_token", C.c_int64), ("causal", C.c_int32), ("window", C.c_int32), ("sink", C.c_int32),
                ("reserved", C.c_int32), ("out", C.c_void_p), ("out_stride_seq", C.c_int64), ("out_stride_head", C.c_int64),
                ("out_stride_token", C.c_int64), ("lse", C.c_void_p)]


class QvgError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def lib():
    """Load libqvg.so (built in-tree by paper_2602_02958_amd.build); raise if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2602_02958_amd.build` "
                "(there is no CPU fallback)")
        L = C.CDLL(_LIB_PATH)
        vp, i64, u8p = C.c_void_p, C.c_int64, C.c_void_p
        pp = C.POINTER(QvgParams)
        L.qvg_encode_chunk.restype = C.c_int
        L.qvg_encode_chunk.argtypes = [pp, i64, vp, i64, i64, vp, vp, i64, u8p, u8p, vp, i64, vp,
                                       C.c_size_t, vp]
        L.qvg_encode_chunk_static.restype = C.c_int
        L.qvg_encode_chunk_static.argtypes = [pp, i64, vp, i64, i64, vp, vp, i64, u8p, u8p, vp, i64, vp]
        L.qvg_decode.restype = C.c_int
        L.qvg_decode.argtypes = [pp, i64, i64, vp, u8p, u8p, vp, vp, i64, i64, vp]
        L.qvg_decode_ex.restype = C.c_int
        L.qvg_decode_ex.argtypes = [pp, i64, i64, i64, i64, vp, u8p, u8p, vp, vp, i64, i64, vp]
        L.qvg_attn_decode.restype = C.c_int
        L.qvg_attn_decode.argtypes = [pp, i64, vp, i64, i64, vp, u8p, u8p, vp, vp, u8p, u8p, vp,
                                      C.c_float, vp, vp, vp, C.c_size_t, vp]
        L.qvg_attn_decode_ex.restype = C.c_int
        L.qvg_attn_decode_ex.argtypes = [pp, i64, vp, i64, i64, i64, vp, u8p, u8p, vp, vp, u8p, u8p, vp, vp,
                                         C.c_float, vp, vp, vp, C.c_size_t, vp]
        L.qvg_attn_decode_causal.restype = C.c_int
        L.qvg_attn_decode_causal.argtypes = [pp, i64, vp, i64, i64, i64, vp, u8p, u8p, vp, vp, u8p, u8p, vp, vp, vp,
                                             C.c_float, vp, vp, vp, C.c_size_t, vp]
        L.qvg_attn_decode_f32.restype = C.c_int
        L.qvg_attn_decode_f32.argtypes = [pp, i64, vp, i64, i64, i64, vp, u8p, u8p, vp, vp, u8p, u8p, vp, vp, vp,
                                          C.c_float, vp, vp, vp]
        L.qvg_attn_decode_parts.restype = C.c_int
        L.qvg_attn_decode_parts.argtypes = [pp, i64, vp, i64, i64, i64, vp, u8p, u8p, vp, vp, u8p, u8p, vp, vp, vp,
                                            C.c_float, vp, vp, vp, vp, C.c_size_t, vp, C.c_size_t, vp]
        L.qvg_attn_scratch_bytes.restype = C.c_int
        L.qvg_attn_scratch_bytes.argtypes = [pp, i64, i64, i64, C.POINTER(C.c_size_t)]
        L.qvg_attn_scratch_bytes_causal.restype = C.c_int
        L.qvg_attn_scratch_bytes_causal.argtypes = L.qvg_attn_scratch_bytes.argtypes
        L.qvg_attn_merge.restype = C.c_int
        L.qvg_attn_merge.argtypes = [i64, C.c_int32, vp, vp, vp, vp, vp, vp, vp]
        pt = C.POINTER(QvgTreeStep)
        L.qvg_attn_tree.restype = C.c_int
        L.qvg_attn_tree.argtypes = [pp, pt, vp, u8p, u8p, vp, vp, u8p, u8p, vp, C.c_float, vp, C.c_size_t, vp]
        L.qvg_attn_tree_scratch_bytes.restype = C.c_int
        L.qvg_attn_tree_scratch_bytes.argtypes = [pp, pt, C.POINTER(C.c_size_t)]
        L.qvg_tree_mask.restype = C.c_int
        L.qvg_tree_mask.argtypes = [i64, i64, vp, vp, vp, vp, vp]
        L.qvg_keep_nodes.restype = C.c_int
        L.qvg_keep_nodes.argtypes = [C.c_int32, C.c_int32, i64, i64, vp, vp, i64, i64, i64, vp, i64, vp, vp, vp, i64, i64, i64,
                                     i64, vp, vp, vp]
        L.qvg_copy_pages.restype = C.c_int
        L.qvg_copy_pages.argtypes = [pp, i64, i64, C.POINTER(C.c_int32), C.POINTER(C.c_int32), i64, vp, u8p, u8p, vp,
                                     i64, vp, u8p, u8p, vp, vp]
        L.qvg_rope_table.restype = C.c_int
        L.qvg_rope_table.argtypes = [i64, C.c_int32, vp, i64, vp, C.c_int32, vp, C.c_float, C.c_int32, vp, vp]
        pr, pc, ps = C.POINTER(QvgRotary), C.POINTER(QvgPageCache), C.POINTER(QvgPageStep)
        L.qvg_rope.restype = C.c_int
        L.qvg_rope.argtypes = [pr, C.c_int32, i64, C.c_int32, i64, C.c_int32, vp, i64, i64, i64, vp, C.c_int32, vp, i64, i64, i64, vp]
        L.qvg_append_pages.restype = C.c_int
        L.qvg_append_pages.argtypes = [pc, i64, vp, vp, i64, i64, i64, vp, pr, vp, vp]
        L.qvg_attn_pages.restype = C.c_int
        L.qvg_attn_pages.argtypes = [pc, ps, C.c_float, vp, C.c_size_t, vp]
        L.qvg_attn_pages_scratch_bytes.restype = C.c_int
        L.qvg_attn_pages_scratch_bytes.argtypes = [pc, ps, C.POINTER(C.c_size_t)]
        L.qvg_kmeans_assign.restype = C.c_int
        L.qvg_kmeans_assign.argtypes = [pp, i64, vp, i64, i64, vp, u8p, vp, C.c_size_t, vp]
        L.qvg_kmeans_update.restype = C.c_int
        L.qvg_kmeans_update.argtypes = [pp, i64, vp, i64, i64, u8p, vp, vp, vp, vp, C.c_size_t, vp]
        L.qvg_workspace_bytes.restype = C.c_int
        L.qvg_workspace_bytes.argtypes = [pp, C.c_int, i64, i64, C.POINTER(C.c_size_t)]
        L.qvg_compressed_bytes.restype = C.c_int64
        L.qvg_compressed_bytes.argtypes = [pp, i64]
        L.qvg_status_string.restype = C.c_char_p
        L.qvg_status_string.argtypes = [C.c_int]
        L.qvg_version.restype = C.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().qvg_status_string(int(status)).decode()


def make_params(n_heads, n_clusters, group_size, n_stages, kmeans_iters=0, head_dim=128, bits=2,
                n_smooth_stages=1, scale_format=SCALE_F16) -> QvgParams:
    return QvgParams(n_heads, head_dim, n_clusters, group_size, n_stages, bits, n_smooth_stages,
                     kmeans_iters, scale_format)


def workspace_bytes(p: QvgParams, entry: int, n_tokens: int, n_q: int = 0) -> int:
    out = C.c_size_t(0)
    st = lib().qvg_workspace_bytes(C.byref(p), entry, n_tokens, n_q, C.byref(out))
    if st != 0:
        raise QvgError(st, "qvg_workspace_bytes")
    return int(out.value)


def compressed_bytes(p: QvgParams, n_tokens: int) -> int:
    v = int(lib().qvg_compressed_bytes(C.byref(p), n_tokens))
    if v < 0:
        raise QvgError(v, "qvg_compressed_bytes")
    return v


def _stream():
    # (torch.cuda.current_stream().cuda_stream without the Stream object, which costs more than all pointers of a call)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _check(t, dtype, name):
    if t.dtype != dtype or not t.is_cuda:
        raise TypeError(f"{name}: expected a cuda tensor of {dtype}, got {t.dtype} on {t.device}")


def _view3(x, name):
    """[H, N, d] bf16 view with a contiguous last dim -> (stride_head, stride_token)."""
    _check(x, torch.bfloat16, name)
    if x.dim() != 3 or x.stride(2) != 1:
        raise ValueError(f"{name}: need [H, N, d] with unit stride along d")
    return x.stride(0), x.stride(1)


@dataclass
class Encoded:
    """Stored form of one chunk (or of a cache of chunks) for H units.  With n_smooth = S > 1
    smoothing stages the tables are [H, n_chunks, S, K, d] and a token has S ids: [H, N, S].
    The formats are read off the tensors: 4-bit levels have d/2 code bytes per round, FP8 E4M3
    scales are a uint8 tensor."""
    centroids: torch.Tensor   # [H, n_chunks, K, d] bf16
    ids: torch.Tensor         # [H, N] uint8 (int16 with more than 256 centroids)
    codes: torch.Tensor       # [H, N, T, d*bits/8] uint8
    scales: torch.Tensor      # [H, N, T, d/B] float16, or uint8 (E4M3)
    chunk_len: int
    n_smooth: int = 1

    @property
    def bits(self) -> int:
        return self.codes.shape[3] * 8 // self.centroids.shape[-1]

    @property
    def scale_format(self) -> int:
        return SCALE_E4M3 if self.scales.dtype == torch.uint8 else SCALE_F16


def id_dtype(n_clusters):
    """Cluster ids are bytes up to 256 centroids and 16-bit words beyond (int16 tensors here: the
    values stay below 512)."""
    return torch.uint8 if n_clusters <= 256 else torch.int16


def _check_stored(cent, ids, codes, scales, K):
    if (cent.dtype is torch.bfloat16 and ids.dtype is id_dtype(K) and codes.dtype is torch.uint8 and
            cent.is_cuda and ids.is_cuda and codes.is_cuda and scales.is_cuda and
            cent.is_contiguous() and ids.is_contiguous() and codes.is_contiguous() and scales.is_contiguous()):
        return
    for t, dt, nm in ((cent, torch.bfloat16, "centroids"), (ids, id_dtype(K), "ids"),
                      (codes, torch.uint8, "codes"), (scales, scales.dtype, "scales")):
        _check(t, dt, nm)
        if not t.is_contiguous():
            raise ValueError(f"{nm} must be contiguous")


def alloc_cache(n_heads, n_tokens, chunk_len, n_clusters, group_size, n_stages, head_dim=128,
                device="cuda", n_smooth=1, bits=2, scale_format=SCALE_F16) -> Encoded:
    """Uninitialised storage for a cache of n_tokens tokens per unit in chunks of chunk_len."""
    n_chunks = max(1, -(-n_tokens // chunk_len))
    S = n_smooth
    cshape = (n_heads, n_chunks, n_clusters, head_dim) if S == 1 else (n_heads, n_chunks, S, n_clusters, head_dim)
    ishape = (n_heads, n_tokens) if S == 1 else (n_heads, n_tokens, S)
    return Encoded(
        torch.empty(cshape, dtype=torch.bfloat16, device=device),
        torch.empty(ishape, dtype=id_dtype(n_clusters), device=device),
        torch.empty(n_heads, n_tokens, n_stages, head_dim * bits // 8, dtype=torch.uint8, device=device),
        torch.empty(n_heads, n_tokens, n_stages, head_dim // group_size,
                    dtype=torch.uint8 if scale_format == SCALE_E4M3 else torch.float16, device=device),
        chunk_len, S)


def encode_chunk(x, init_centroids, group_size, n_stages, kmeans_iters, cache: Encoded | None = None,
                 chunk_index: int = 0, workspace=None, bits=2, scale_format=SCALE_F16,
                 static_scratch: bool = False) -> Encoded:
    """qvg_encode_chunk.  x [H, N, d] bf16, init_centroids [H, K, d] bf16, or [H, S, K, d] for S
    smoothing stages.  Without `cache` a one-chunk cache is allocated and returned; with it, the
    chunk is written in place at chunk_index (tokens chunk_index*chunk_len ...), using the output
    strides; the cache's formats then apply (bits and scale_format describe a new cache).
    static_scratch: call qvg_encode_chunk_static instead (no workspace: the library's own static
    scratch array; with a `cache` given the call allocates nothing at all)."""
    sh, st_ = _view3(x, "x")
    H, N, d = x.shape
    _check(init_centroids, torch.bfloat16, "init_centroids")
    init_centroids = init_centroids.contiguous()
    K = init_centroids.shape[-2]
    S = init_centroids.shape[1] if init_centroids.dim() == 4 else 1
    if cache is None:
        cache = alloc_cache(H, N, max(N, 1), K, group_size, n_stages, d, x.device, n_smooth=S, bits=bits,
                            scale_format=scale_format)
    bits, scale_format = cache.bits, cache.scale_format
    n_total = cache.ids.shape[1]
    n_chunks = cache.centroids.shape[1]
    off = chunk_index * cache.chunk_len
    if not (0 <= chunk_index < n_chunks) or off + N > n_total or (N > cache.chunk_len):
        raise ValueError("chunk does not fit the cache")
    if cache.codes.shape[2] != n_stages or cache.scales.shape[3] != d // group_size or \
            cache.centroids.shape[-2] != K or cache.ids.shape[0] != H or cache.n_smooth != S or \
            cache.ids.dtype != id_dtype(K):
        raise ValueError("cache was allocated for other parameters")
    p = make_params(H, K, group_size, n_stages, kmeans_iters, head_dim=d, n_smooth_stages=S, bits=bits,
                    scale_format=scale_format)
    T, G = n_stages, d // group_size
    outs = (cache.centroids.data_ptr() + chunk_index * S * K * d * 2, n_chunks * S * K * d,
            cache.ids.data_ptr() + off * S * cache.ids.element_size(),
            cache.codes.data_ptr() + off * T * (d * bits // 8),
            cache.scales.data_ptr() + off * T * G * cache.scales.element_size(), n_total)
    if static_scratch:
        st = lib().qvg_encode_chunk_static(C.byref(p), N, _ptr(x), sh, st_, _ptr(init_centroids), *outs, _stream())
        if st != 0:
            raise QvgError(st, "qvg_encode_chunk_static")
        return cache
    need = workspace_bytes(p, ENTRY_ENCODE, N)
    if need and (workspace is None or workspace.numel() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    st = lib().qvg_encode_chunk(C.byref(p), N, _ptr(x), sh, st_, _ptr(init_centroids), *outs,
                                _ptr(workspace) if need else None, need, _stream())
    if st != 0:
        raise QvgError(st, "qvg_encode_chunk")
    return cache


def decode(enc: Encoded, out=None, n_tokens=None, first_token=0) -> torch.Tensor:
    """qvg_decode_ex -> bf16 [H, n_tokens, d]: the whole cache, or n_tokens tokens starting at
    first_token (a multiple of the chunk length)."""
    cent, ids, codes, scales = enc.centroids, enc.ids, enc.codes, enc.scales
    H, cap = ids.shape[:2]
    N = cap - first_token if n_tokens is None else int(n_tokens)
    if first_token < 0 or N < 0 or first_token + N > cap:
        raise ValueError("token range outside the cache")
    K, d = cent.shape[-2:]
    T, code_bytes = codes.shape[2:]
    p = QvgParams(H, d, K, d // scales.shape[3], T, code_bytes * 8 // d, enc.n_smooth, 0, enc.scale_format)
    if out is None:
        out = torch.empty(H, N, d, dtype=torch.bfloat16, device=ids.device)
    sh, st_ = _view3(out, "out")
    _check_stored(cent, ids, codes, scales, K)
    st = lib().qvg_decode_ex(p, N, enc.chunk_len, cap, first_token, cent.data_ptr(), ids.data_ptr(), codes.data_ptr(),
                             scales.data_ptr(), out.data_ptr(), sh, st_, _stream())
    if st != 0:
        raise QvgError(st, "qvg_decode_ex")
    return out


def attn_workspace(heads: int, n_q: int, chunk_len: int, n_chunks: int, device) -> torch.Tensor:
    """A workspace for attn_decode that holds the decoded tiles of n_chunks chunks (and the
    queries' running state, which is used when the cache has more chunks than that)."""
    p = make_params(heads, 2, 128, 1)
    padded = -(-chunk_len // 64) * 64 * n_chunks
    return torch.empty(workspace_bytes(p, ENTRY_ATTN, padded, n_q), dtype=torch.uint8, device=device)


def _scratch(nbytes: int, device):
    """Scratch of one call, from torch's allocator on the current stream; None when there is none to be
    had (the library then takes the form that needs none)."""
    if nbytes == 0:
        return None
    try:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    except torch.OutOfMemoryError:
        return None


def _may_divide(n_kv, chunk_len):
    """False for caches of fewer than four tiles, which are never divided: a call over them is host time and does without
    the question (which a call of sizes that were not there before puts to the library)."""
    return n_kv // 64 + n_kv // chunk_len >= 3


@functools.lru_cache(maxsize=256)
def _parts_bytes(H, d, K, group_size, T, bits, n_smooth, scale_format, n_q, n_kv, chunk_len, with_len) -> int:
    """Bytes of scratch that let a call of these sizes be divided: a function of its arguments alone, so a call like
    the one before does not ask the library again."""
    need = C.c_size_t()
    ask = lib().qvg_attn_scratch_bytes_causal if with_len else lib().qvg_attn_scratch_bytes
    st = ask(QvgParams(H, d, K, group_size, T, bits, n_smooth, 0, scale_format), n_q, n_kv, chunk_len, C.byref(need))
    if st != 0:
        raise QvgError(st, "qvg_attn_scratch_bytes")
    return need.value


# An attn_decode that is lent no workspace takes one for itself when a unit has three query blocks or more:
# 40 heads over 31997 tokens, 900 queries 2.90 -> 1.10 ms, 12 heads x 600 queries over 20000 195 -> 170 us; with two
# blocks the one-kernel form is as fast or faster (40 heads x 300 queries over 20000 305 against 418 us).
# Not with a prefix length per query: the workspace decodes every tile of the cache, however short the prefixes
# (which only the device knows), the one-kernel form those below the longest (12 heads x 600 queries that see
# 300 of 74880 tokens: 235 us with one, 26 without).
# Nor over fewer than four tiles: 700 queries of 1, 12 or 40 heads over 64 tokens 17 us with one, 12.5 without; over 256
# 19 against 21 (40 heads: 22.8 against 21.9).
TILE_SCRATCH_MIN_QUERIES = 512
TILE_SCRATCH_MIN_TOKENS = 256
TILE_SCRATCH_TILES = 256 << 20       # bytes of decoded tiles: a slab
TILE_SCRATCH_STATE = 256 << 20       # bytes of running state (528 per query and head), where one slab is not the whole cache


def _tile_scratch_bytes(heads, n_q, chunk_len, n_chunks):
    """Bytes of the workspace of an attn_decode that was lent none: the whole cache where it fits
    TILE_SCRATCH_TILES, else the running state and as many chunks as fit; 0 (none) when not even one does,
    or when the state alone is larger than TILE_SCRATCH_STATE."""
    one = heads * -(-chunk_len // 64) * 64 * 512
    chunks = min(n_chunks, TILE_SCRATCH_TILES // one)
    if chunks == n_chunks:
        return one * chunks
    state = workspace_bytes(make_params(heads, 2, 128, 1), ENTRY_ATTN, 0, n_q)
    return one * chunks + state if chunks > 0 and state <= TILE_SCRATCH_STATE else 0


def attn_decode(q, k: Encoded, v: Encoded, softmax_scale=None, want_lse=False, out=None, n_kv=None,
                k_rope=None, q_kv_len=None, f32_out=False, workspace=None):
    """qvg_attn_decode_parts.  q [H, Nq, d] bf16 contiguous -> out bf16 [H, Nq, d] (and lse fp32 [H, Nq]).
    n_kv: read only the first n_kv tokens of the caches (they are allocated for more);
    k_rope: [n_kv, d/2, 2] float16 (cos, sin), the rotary embedding of the decoded keys;
    q_kv_len: [Nq] int32, query i sees the first q_kv_len[i] tokens only;
    f32_out: the result as float32, before the rounding to bf16;
    workspace: uint8 tensor (attn_workspace): every tile is then decoded once per unit into it and
    shared by all query blocks, a slab of chunks at a time, instead of once per 256 queries.  Without
    one, calls of more than 512 queries over 256 tokens or more, without q_kv_len, take it from torch's allocator for the call: up to
    256 MiB of tiles, and up to 256 MiB of running state when the cache needs more.  One that is too
    small for a chunk (an empty tensor) is ignored.  Worth lending with q_kv_len too, unless the prefixes
    are short: every tile of the cache is decoded.  Calls of few query blocks, or with up to 128 beyond a multiple of 256, take up to 34 MiB for the
    partial results of their divided cache, with q_kv_len calls of up to 256 blocks of 256 queries up to 99 MiB; where torch has no memory left they run undivided, which
    differs by the order of fp32 sums."""
    if (v.ids.shape, v.codes.shape, v.scales.shape, v.scales.dtype, v.centroids.shape, v.chunk_len, v.n_smooth) != \
            (k.ids.shape, k.codes.shape, k.scales.shape, k.scales.dtype, k.centroids.shape, k.chunk_len, k.n_smooth):
        raise ValueError("K and V caches must share shapes and parameters")
    _check(v.ids, id_dtype(v.centroids.shape[-2]), "v.ids")
    kp = (_ptr(k.centroids), _ptr(k.ids), _ptr(k.codes), _ptr(k.scales))
    vp = (_ptr(v.centroids), _ptr(v.ids), _ptr(v.codes), _ptr(v.scales))
    return _attn(q, k, kp, vp, softmax_scale, want_lse, out, n_kv, k_rope, q_kv_len, f32_out, workspace)


def _attn(q, k: Encoded, kp, vp, softmax_scale, want_lse, out, n_kv, k_rope, q_kv_len, f32_out, workspace):
    """attn_decode on the pointers kp and vp (centroids, ids, codes, scales of the two sides); sizes and
    formats are those of k."""
    _check(q, torch.bfloat16, "q")
    q = q.contiguous()
    H, Nq, d = q.shape
    cap = k.ids.shape[1]
    Nk = cap if n_kv is None else int(n_kv)
    if not (1 <= Nk <= cap):
        raise ValueError("n_kv must lie in 1 .. the caches' token capacity")
    if k_rope is not None:
        _check(k_rope, torch.float16, "k_rope")
        if tuple(k_rope.shape) != (Nk, d // 2, 2) or not k_rope.is_contiguous():
            raise ValueError("k_rope: need a contiguous [n_kv, d/2, 2] float16 tensor")
    K = k.centroids.shape[-2]
    T, code_bytes = k.codes.shape[2:]
    G = k.scales.shape[3]
    _check(k.ids, id_dtype(K), "k.ids")
    p = QvgParams(H, d, K, d // G, T, code_bytes * 8 // d, k.n_smooth, 0, k.scale_format)
    if softmax_scale is None:
        softmax_scale = 1.0 / (d ** 0.5)
    if out is None:
        out = torch.empty(H, Nq, d, dtype=torch.float32 if f32_out else torch.bfloat16, device=q.device)
    lse = torch.empty(H, Nq, dtype=torch.float32, device=q.device) if want_lse else None
    if q_kv_len is not None:
        _check(q_kv_len, torch.int32, "q_kv_len")
        if tuple(q_kv_len.shape) != (Nq,) or not q_kv_len.is_contiguous():
            raise ValueError("q_kv_len: need a contiguous [n_q] int32 tensor")
    if f32_out:
        _check(out, torch.float32, "out")
        if not out.is_contiguous():
            raise ValueError("out must be contiguous")
    scratch = None
    if _may_divide(Nk, k.chunk_len):
        scratch = _scratch(_parts_bytes(H, d, K, d // G, T, p.bits, k.n_smooth, p.scale_format, Nq, Nk, k.chunk_len,
                                        q_kv_len is not None), q.device)
    if workspace is None and q_kv_len is None and Nq > TILE_SCRATCH_MIN_QUERIES and Nk >= TILE_SCRATCH_MIN_TOKENS:
        workspace = _scratch(_tile_scratch_bytes(H, Nq, k.chunk_len, -(-Nk // k.chunk_len)), q.device)
    st = lib().qvg_attn_decode_parts(C.byref(p), Nq, _ptr(q), Nk, k.chunk_len, cap,
                                     *kp, *vp, _ptr(k_rope), _ptr(q_kv_len), softmax_scale,
                                     None if f32_out else _ptr(out), _ptr(out) if f32_out else None, _ptr(lse),
                                     _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                     _ptr(scratch), 0 if scratch is None else scratch.numel(), _stream())
    if st != 0:
        raise QvgError(st, "qvg_attn_decode_parts")
    return (out, lse) if want_lse else out


def attn_merge(out_a, lse_a, out_b, lse_b, out=None, want_lse=False):
    """qvg_attn_merge.  out_* bf16 [..., d] contiguous, lse_* fp32 [...] -> merged bf16 (and lse)."""
    for t, dt, nm in ((out_a, torch.bfloat16, "out_a"), (out_b, torch.bfloat16, "out_b"),
                      (lse_a, torch.float32, "lse_a"), (lse_b, torch.float32, "lse_b")):
        _check(t, dt, nm)
        if not t.is_contiguous():
            raise ValueError(f"{nm} must be contiguous")
    d = out_a.shape[-1]
    rows = out_a.numel() // d
    if out_b.shape != out_a.shape or lse_a.numel() != rows or lse_b.numel() != rows:
        raise ValueError("shapes of the two partial results differ")
    if out is None:
        out = torch.empty_like(out_a)
    lse = torch.empty_like(lse_a) if want_lse else None
    st = lib().qvg_attn_merge(rows, d, _ptr(out_a), _ptr(lse_a), _ptr(out_b), _ptr(lse_b), _ptr(out), _ptr(lse),
                              _stream())
    if st != 0:
        raise QvgError(st, "qvg_attn_merge")
    return (out, lse) if want_lse else out


def _rows4(x, name, shape=None):
    """[B, H, N, d] bf16 view with a contiguous last dim -> its three strides (of a dimension of one element 0: it is not
    used, and a view may hold anything there)."""
    if x.dtype is not torch.bfloat16 or not x.is_cuda:
        _check(x, torch.bfloat16, name)
    if x.dim() != 4 or x.stride(3) != 1 or (shape is not None and x.shape != shape):
        raise ValueError(f"{name}: need bf16 {'[B, H, N, d]' if shape is None else list(shape)} with unit stride along d")
    a, b, c, _ = x.stride()
    if (a | b | c) & 7:
        return tuple(0 if n == 1 else s for n, s in zip(x.shape[:3], (a, b, c)))
    return a, b, c


def _same_rows(x, y, names, shape=None):
    """The strides that two views share."""
    sx, sy = _rows4(x, names[0], shape), _rows4(y, names[1], x.shape)
    if sx != sy and any(a != b and n != 1 for a, b, n in zip(sx, sy, x.shape)):
        raise ValueError(f"{names[0]} and {names[1]} must share their strides")
    return sx


def _ints(t, shape, name):
    if t.dtype is not torch.int32 or not t.is_cuda:
        _check(t, torch.int32, name)
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: need a contiguous int32 tensor of shape {list(shape)}")
    return t.data_ptr()


def _here(*tensors):
    """All tensors of a call are on the current device: its stream is the one the call goes to."""
    dev = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{dev}")


def _check_arrays(e: Encoded, K):
    """A pool's arrays, all on one device (cheaper than asking each of them twice); returns it."""
    cent, ids, codes, scales = e.centroids, e.ids, e.codes, e.scales
    at = ids.get_device()
    if not (cent.dtype is torch.bfloat16 and ids.dtype is id_dtype(K) and codes.dtype is torch.uint8 and
            at >= 0 and cent.get_device() == at and codes.get_device() == at and scales.get_device() == at and
            cent.is_contiguous() and ids.is_contiguous() and codes.is_contiguous() and scales.is_contiguous()):
        _check_stored(cent, ids, codes, scales, K)
        _here(cent, ids, codes, scales)
    return at


def _check_pool(e: Encoded, name):
    """The arrays of a pool agree with each other: whole pages, a set of tables to each.  Returns (units, pages, K, d)."""
    cent, S, L = e.centroids.shape, e.n_smooth, e.chunk_len
    units, tokens, T, _ = e.codes.shape
    s_units, s_tokens, s_T, _ = e.scales.shape
    pages = tokens // L
    if pages * L != tokens or pages < 1:
        raise ValueError(f"{name}: the pool must hold whole pages of {L} tokens")
    if (units != s_units or tokens != s_tokens or T != s_T or cent[:-2] != ((units, pages) if S == 1 else (units, pages, S)) or
            e.ids.shape != ((units, tokens) if S == 1 else (units, tokens, S))):
        raise ValueError(f"{name}: the pool's arrays are of different sizes")
    K, d = cent[-2:]
    _check_arrays(e, K)
    return units, pages, K, d


@functools.lru_cache(maxsize=256)
def _tree_scratch_bytes(H, group_size, T, bits, n_smooth, scale_format, n_seqs, group, n_nodes, table_pages, page_len, tail_capacity) -> int:
    """Bytes of scratch of an attn_tree of these sizes (a function of its arguments alone)."""
    need = C.c_size_t()
    t = QvgTreeStep(n_seqs=n_seqs, group=group, n_nodes=n_nodes, table_pages=table_pages, page_len=page_len, pool_pages=1,
                    tail_capacity=tail_capacity)
    st = lib().qvg_attn_tree_scratch_bytes(QvgParams(H, 128, 2, group_size, T, bits, n_smooth, 0, scale_format), C.byref(t), C.byref(need))
    if st != 0:
        raise QvgError(st, "qvg_attn_tree_scratch_bytes")
    return need.value


def tree_mask(parents, n_nodes=None, mask=None, depth=None):
    """qvg_tree_mask.  parents [B, N] int32 (the parent of node i, below i; -1: none) -> (mask [B, N, ceil(N / 32)] int32,
    depth [B, N] int32).  n_nodes [B] int32: a tree's nodes, all N without.  Nodes behind them, and those with another
    parent than allowed, are holes: an empty row, depth -1."""
    _check(parents, torch.int32, "parents")
    if parents.dim() != 2 or not parents.is_contiguous():
        raise ValueError("parents: need a contiguous [B, N] int32 tensor")
    _here(parents, n_nodes, mask, depth)
    n, m = parents.shape
    words = -(-m // 32)
    mask = torch.empty(n, m, words, dtype=torch.int32, device=parents.device) if mask is None else mask
    depth = torch.empty(n, m, dtype=torch.int32, device=parents.device) if depth is None else depth
    st = lib().qvg_tree_mask(n, m, parents.data_ptr(), None if n_nodes is None else _ints(n_nodes, (n,), "n_nodes"),
                             _ints(mask, (n, m, words), "mask"), _ints(depth, (n, m), "depth"), _stream())
    if st != 0:
        raise QvgError(st, "qvg_tree_mask")
    return mask, depth


def attn_tree(q, k: Encoded, v: Encoded, page_table, kv_len, k_new, v_new, tail_k=None, tail_v=None, tail_len=None, n_nodes=None,
              mask=None, softmax_scale=None, k_rope=None, want_lse=False, out=None, scratch=None):
    """qvg_attn_tree: attention of the new tokens of B sequences over their compressed pages, their bf16 tails and each other.
    q [B, H * group, N, d] bf16 -> out [B, H * group, N, d] (and lse fp32 [B, H * group, N]); query head h reads KV head
    h // group.
    k, v: the pools, [H] units of pages of chunk_len tokens (alloc_cache, filled by encode_chunk: chunk_index is the page);
    page_table [B, P] int32, kv_len [B] int32: the sequences' pages and how many tokens they hold (page_table None: none);
    k_new, v_new [B, H, N, d] bf16: the new tokens' own K and V; n_nodes [B] int32: how many there are (None: N);
    mask [B, N, ceil(N / 32)] int32 (tree_mask): which new tokens a new token sees (None: itself and those before it);
    tail_k, tail_v [B, H, R, d] bf16, tail_len [B] int32: tokens that are in no page yet;
    k_rope [n, d/2, 2] float16: rotary embedding of the compressed keys by their place in the sequence.
    Views may be strided (multiples of 8 elements, unit stride along d); K and V views share their strides.  Rows behind
    n_nodes, and those that see nothing, are zero with lse -inf.
    scratch: uint8 tensor of attn_tree_scratch bytes for dividing the call over the chip; without one it is taken from torch's
    allocator (where that has no memory left the call runs undivided, which differs by the order of fp32 sums)."""
    if (v.ids.shape, v.codes.shape, v.scales.shape, v.scales.dtype, v.centroids.shape, v.chunk_len, v.n_smooth) != \
            (k.ids.shape, k.codes.shape, k.scales.shape, k.scales.dtype, k.centroids.shape, k.chunk_len, k.n_smooth):
        raise ValueError("K and V pools must share shapes and parameters")
    _check_pool(k, "k")
    if _check_arrays(v, v.centroids.shape[-2]) != k.ids.get_device():                    # (the shapes are k's)
        _here(k.ids, v.ids)
    return _attn_tree(q, k, (k.centroids.data_ptr(), k.ids.data_ptr(), k.codes.data_ptr(), k.scales.data_ptr()),
                      (v.centroids.data_ptr(), v.ids.data_ptr(), v.codes.data_ptr(), v.scales.data_ptr()), k.ids.shape[0], page_table,
                      kv_len, k_new, v_new, tail_k, tail_v, tail_len, n_nodes, mask, softmax_scale, k_rope, want_lse, out, scratch)


def attn_tree_scratch(k: Encoded, n_seqs, group, n_nodes, table_pages, tail_capacity) -> torch.Tensor:
    """Scratch for an attn_tree of these sizes over the pool k."""
    _, _, T, code_bytes = k.codes.shape
    d = k.centroids.shape[-1]
    return torch.empty(_tree_scratch_bytes(k.ids.shape[0], d // k.scales.shape[3], T, code_bytes * 8 // d, k.n_smooth, k.scale_format,
                                           n_seqs, group, n_nodes, table_pages, k.chunk_len, tail_capacity),
                       dtype=torch.uint8, device=k.ids.device)


def _attn_tree(q, k: Encoded, kp, vp, H, page_table, kv_len, k_new, v_new, tail_k, tail_v, tail_len, n_nodes, mask,
               softmax_scale, k_rope, want_lse, out, scratch):
    """attn_tree on the pointers kp and vp (centroids, ids, codes, scales of the two pools) of H units each; sizes and formats
    are those of k."""
    qs = _rows4(q, "q")
    n, hq, m, d = q.shape
    if hq < H or hq % H:
        raise ValueError("q: the number of query heads must be a multiple of the KV heads'")
    K, pool_d = k.centroids.shape[-2:]
    if pool_d != d:
        raise ValueError(f"q: the pools hold heads of {pool_d} channels")
    _, _, T, code_bytes = k.codes.shape
    L = k.chunk_len
    ns = _same_rows(k_new, v_new, ("k_new", "v_new"), (n, H, m, d))
    _here(q, k.ids, k_new, v_new, page_table, kv_len, tail_k, tail_v, tail_len, n_nodes, mask, k_rope, out, scratch)
    pages, table, lens, rope, rope_tokens = 0, None, None, None, 0
    if page_table is not None and page_table.shape[-1] > 0:
        pages = page_table.shape[-1]
        table, lens = _ints(page_table, (n, pages), "page_table"), _ints(kv_len, (n,), "kv_len")
        if k_rope is not None:
            _check(k_rope, torch.float16, "k_rope")
            if k_rope.dim() != 3 or k_rope.shape[1:] != (d // 2, 2) or not k_rope.is_contiguous() or k_rope.shape[0] < 1:
                raise ValueError("k_rope: need a contiguous [n, d/2, 2] float16 tensor")
            rope, rope_tokens = k_rope.data_ptr(), k_rope.shape[0]
    R, tail, ts = 0, (None, None, None), (0, 0, 0)
    if tail_k is not None and tail_k.shape[2] > 0:
        if tail_v is None or tail_len is None:
            raise ValueError("tail_k needs tail_v and tail_len")
        R = tail_k.shape[2]
        ts = _same_rows(tail_k, tail_v, ("tail_k", "tail_v"), (n, H, R, d))
        tail = (tail_k.data_ptr(), tail_v.data_ptr(), _ints(tail_len, (n,), "tail_len"))
    if out is None:
        out = torch.empty(n, hq, m, d, dtype=torch.bfloat16, device=q.device)
        os_ = (hq * m * d, m * d, d)
    else:
        os_ = _rows4(out, "out", q.shape)
    lse = torch.empty(n, hq, m, dtype=torch.float32, device=q.device) if want_lse else None
    B, bits, fp8 = d // k.scales.shape[3], code_bytes * 8 // d, k.scale_format
    if scratch is not None:
        if scratch.dtype is not torch.uint8 or not scratch.is_contiguous():
            raise ValueError("scratch: need a contiguous uint8 tensor")
    else:
        scratch = _scratch(_tree_scratch_bytes(H, B, T, bits, k.n_smooth, fp8, n, hq // H, m, pages, L, R), q.device)
    # (fields in the struct's order: naming them costs more than the smallest call's launches)
    t = QvgTreeStep(n, hq // H, m, pages, L, max(1, k.ids.shape[1] // L), table, lens, q.data_ptr(), *qs,
                    k_new.data_ptr(), v_new.data_ptr(), *ns, tail[0], tail[1], *ts, tail[2], R, 0,
                    None if n_nodes is None else _ints(n_nodes, (n,), "n_nodes"),
                    None if mask is None else _ints(mask, (n, m, -(-m // 32)), "mask"), rope, rope_tokens, out.data_ptr(), *os_, _ptr(lse))
    p = QvgParams(H, d, K, B, T, bits, k.n_smooth, 0, fp8)
    st = lib().qvg_attn_tree(p, C.byref(t), *kp, *vp, 1.0 / (d ** 0.5) if softmax_scale is None else softmax_scale,
                             _ptr(scratch), 0 if scratch is None else scratch.numel(), _stream())
    if st != 0:
        raise QvgError(st, "qvg_attn_tree")
    return (out, lse) if want_lse else out


def keep_nodes(k_new, v_new, path, n_keep, tail_k, tail_v, tail_len, out_len=None) -> torch.Tensor:
    """qvg_keep_nodes: the K and V of the kept new tokens go behind the tails.  k_new, v_new [B, H, N, d] bf16; path [B, M] int32:
    the kept tokens' indices in order, n_keep [B] int32 how many; tail_k, tail_v [B, H, R, d] bf16 (written in place),
    tail_len [B] int32.  Returns the new lengths [B] int32 (out_len, which may be tail_len itself, or a new tensor)."""
    ns = _same_rows(k_new, v_new, ("k_new", "v_new"))
    n, H, m, d = k_new.shape
    ts = _same_rows(tail_k, tail_v, ("tail_k", "tail_v"), (n, H, tail_k.shape[2], d) if tail_k.dim() == 4 else None)
    if path.dim() != 2:
        raise ValueError("path: need [B, M]")
    _here(k_new, v_new, path, n_keep, tail_k, tail_v, tail_len, out_len)
    out_len = torch.empty_like(tail_len) if out_len is None else out_len
    st = lib().qvg_keep_nodes(H, d, n, m, k_new.data_ptr(), v_new.data_ptr(), *ns, _ints(path, (n, path.shape[1]), "path"), path.shape[1],
                              _ints(n_keep, (n,), "n_keep"), tail_k.data_ptr(), tail_v.data_ptr(), *ts, tail_k.shape[2],
                              _ints(tail_len, (n,), "tail_len"), _ints(out_len, (n,), "out_len"), _stream())
    if st != 0:
        raise QvgError(st, "qvg_keep_nodes")
    return out_len


def copy_pages(cache: Encoded, src, dst, into: Encoded | None = None) -> Encoded:
    """qvg_copy_pages: page src[i] of every unit of the pool `cache` becomes page dst[i] of the pool `into` (the same one
    without).  src, dst: sequences of Python integers; no destination twice, and none that is a source in the same pool."""
    into = cache if into is None else into
    if into is not cache and (into.chunk_len, into.n_smooth, into.ids.shape[0], into.codes.shape[2:], into.scales.shape[2:], into.scales.dtype,
                              into.centroids.shape[2:]) != (cache.chunk_len, cache.n_smooth, cache.ids.shape[0], cache.codes.shape[2:],
                                                            cache.scales.shape[2:], cache.scales.dtype, cache.centroids.shape[2:]):
        raise ValueError("the pools were allocated for different parameters")
    if len(src) != len(dst):
        raise ValueError("src and dst must have the same length")
    L = cache.chunk_len
    units, pages, K, d = _check_pool(cache, "cache")
    into_pages = pages if into is cache else _check_pool(into, "into")[1]
    _here(cache.ids, into.ids)
    T, code_bytes = cache.codes.shape[2:]
    p = QvgParams(units, d, K, d // cache.scales.shape[3], T, code_bytes * 8 // d, cache.n_smooth, 0, cache.scale_format)
    ints = C.c_int32 * len(src)
    ptrs = [(n, c.centroids.data_ptr(), c.ids.data_ptr(), c.codes.data_ptr(), c.scales.data_ptr()) for n, c in ((pages, cache), (into_pages, into))]
    # (array: a number that does not fit 32 bits is an error, not another page)
    st = lib().qvg_copy_pages(p, L, len(src), ints.from_buffer(array("i", src)), ints.from_buffer(array("i", dst)), *ptrs[0], *ptrs[1],
                              _stream())
    if st != 0:
        raise QvgError(st, "qvg_copy_pages")
    return into


def rope_frequencies(rotary_dim, base=10000.0, scaling=None, factor=1.0, trained=None, low=1.0, high=32.0, device="cuda"):
    """Frequencies of a rotary embedding of `rotary_dim` channels and the amplitude that goes with them: (float64 [rotary_dim / 2],
    float), base^(-2p / rotary_dim) radians a place.  For contexts `factor` times as long as those trained with:
    scaling "linear": every frequency divided by factor (positional interpolation, Chen et al. 2023);
    "base": the base raised to base * factor^(r / (r - 2)), r = rotary_dim: the slowest pair is divided by factor, the fastest one stays
    (known as NTK-aware scaling);
    "bands": by the number of turns a pair makes in `trained` places: from `high` on as it is, below `low` divided by factor, between
    them mixed in proportion; amplitude 0.1 ln(factor) + 1, which both sides of a score are multiplied by (YaRN, Peng et al. 2023)."""
    if rotary_dim < 2 or rotary_dim % 2:
        raise ValueError("rotary_dim: need an even number of channels")
    if not (base > 0 and math.isfinite(base) and factor >= 1 and math.isfinite(factor)):
        raise ValueError("base and factor: need finite numbers, base > 0 and factor >= 1")
    n, amplitude = rotary_dim // 2, 1.0
    if scaling == "base":
        if n < 2:
            raise ValueError("a single pair has no base to raise")
        base *= factor ** (rotary_dim / (rotary_dim - 2))
    f = [base ** (-p / n) for p in range(n)]
    if scaling == "linear":
        f = [x / factor for x in f]
    elif scaling == "bands":
        if trained is None or trained < 1 or not 0 <= low < high:
            raise ValueError("bands: need the places trained with, and 0 <= low < high")
        keep = [min(max((trained * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for x in f]
        f = [x * (k + (1 - k) / factor) for x, k in zip(f, keep)]
        amplitude = 0.1 * math.log(factor) + 1.0
    elif scaling not in (None, "base"):
        raise ValueError(f"scaling: {scaling!r} is not one of None, 'linear', 'base', 'bands'")
    return torch.tensor(f, dtype=torch.float64, device=device), amplitude


def rope_table(n, frequencies, first=0, positions=None, axis=None, amplitude=1.0, dtype=torch.float16, out=None) -> torch.Tensor:
    """qvg_rope_table -> [n, P, 2] (cos, sin), float16 (what the attention over compressed keys reads) or float32.  frequencies [P]
    float64 (rope_frequencies), radians a place.  Row i is place first + i, or positions [n, A] int32 holds its place on each of A
    axes (the frame, row and column of a video's token); axis: the axis of each pair, P Python integers (None: 0)."""
    _check(frequencies, torch.float64, "frequencies")
    if frequencies.dim() != 1 or not frequencies.is_contiguous():
        raise ValueError("frequencies: need a contiguous [P] tensor")
    if dtype not in (torch.float16, torch.float32):
        raise TypeError("a table is float16 or float32")
    P, A, pos, ax = frequencies.shape[0], 1, None, None
    if positions is not None:
        if positions.dim() != 2:
            raise ValueError("positions: need [n, A]")
        A = positions.shape[1]
        pos = _ints(positions, (n, A), "positions")
    if axis is not None:
        if len(axis) != P:
            raise ValueError(f"axis: need the axes of {P} pairs")
        ax = (C.c_int32 * P).from_buffer(array("i", axis))               # (array: a number that does not fit 32 bits is an error)
    if out is None:
        out = torch.empty(n, P, 2, dtype=dtype, device=frequencies.device)
    elif out.shape != (n, P, 2) or not out.is_contiguous():
        raise ValueError(f"out: need a contiguous [{n}, {P}, 2] tensor")
    else:
        _check(out, dtype, "out")
        torch.autograd.graph.increment_version(out)                      # (a gradient of rope that has kept it is an error then)
    _here(frequencies, positions, out)
    first = max(min(first, 1 << 31), -1)                                 # (ctypes keeps the low bits only)
    st = lib().qvg_rope_table(n, P, frequencies.data_ptr(), first, pos, A, ax, amplitude, TYPES[dtype], out.data_ptr(), _stream())
    if st != 0:
        raise QvgError(st, "qvg_rope_table")
    return out


# What the calls below check is asked for at a glance, one tensor's attribute once, and one by one only to say what is wrong: the
# smallest call's launches cost less than asking (append_pages of one token to each of 64 sequences 15.5 -> 14.3 us so).
def _all_here(*tensors):
    """All tensors of a call are on the current device."""
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            break
    else:
        if dev >= 0 and dev == torch._C._cuda_getDevice():
            return
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise TypeError(f"expected cuda tensors, got one of {t.dtype} on {t.device}")
    _here(*tensors)


def _rows_of(x, name, dtype=None, shape=None, written=False):
    """[B, H, N, d] view with a contiguous last dim -> its strides (of a dimension of one element 0 where they break the alignment
    rule, as in _rows4)."""
    have, strides = x.shape, x.stride()
    if x.dtype is not dtype if dtype is not None else x.dtype not in TYPES:
        raise TypeError(f"{name}: expected a tensor of {dtype or 'bfloat16, float16 or float32'}, got {x.dtype}")
    if len(have) != 4 or (shape is not None and have != shape) or strides[3] != 1:
        raise ValueError(f"{name}: need {'[B, H, N, d]' if shape is None else list(shape)} with unit stride along d")
    a, b, c, _ = strides
    if written and not (a and b and c) and any(s == 0 and n > 1 for s, n in zip(strides, have[:3])):
        raise ValueError(f"{name}: rows that are written lie in places of their own")
    if (a | b | c) & 7:
        return tuple(0 if n == 1 else s for n, s in zip(have, strides))
    return strides


def _two_rows(x, y, names, dtype=None, written=False):
    """Two views of one shape and type -> the strides that they share."""
    s, shape = x.stride(), x.shape
    if (y.stride() == s and y.shape == shape and x.dtype is dtype and y.dtype is dtype and len(shape) == 4 and s[3] == 1 and s[0] and s[1] and s[2] and
            not (s[0] | s[1] | s[2]) & 7):
        return s
    sx, sy = _rows_of(x, names[0], dtype, None, written), _rows_of(y, names[1], x.dtype, shape, written)
    _same_strides(sx, sy, shape, names)
    return sx


def _same_strides(sx, sy, shape, names):
    if sx != sy and any(a != b and n != 1 for a, b, n in zip(sx, sy, shape)):
        raise ValueError(f"{names[0]} and {names[1]} must share their strides")


def _counts(t, shape, name):
    """The address of a contiguous int32 tensor."""
    if t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous():
        if t.dtype is not torch.int32:
            raise TypeError(f"{name}: expected a tensor of torch.int32, got {t.dtype}")
        raise ValueError(f"{name}: need a contiguous int32 tensor of shape {list(shape)}")
    return t.data_ptr()


def _rotary(table, half, positions, shape) -> QvgRotary:
    kind, have = table.dtype, table.shape
    if kind is not torch.float16 and kind is not torch.float32:
        raise TypeError(f"a rotary table is a float16 or float32 tensor, got {kind}")
    if len(have) != 3 or have[2] != 2 or have[0] < 1 or not table.is_contiguous():
        raise ValueError("a rotary table is a contiguous [n, P, 2] tensor")
    return QvgRotary(table.data_ptr(), TYPES[kind], have[1], have[0], 1 if half else 0, 0, None if positions is None else _counts(positions, shape, "positions"))


def rope(x, table, positions=None, first=None, half=False, backward=False, out=None) -> torch.Tensor:
    """qvg_rope: rows of x [B, H, N, d] (bf16, float16 or float32) turned by a table [n, P, 2] (rope_table): the first 2P of their channels
    in pairs (2p, 2p + 1), or with half=True (p, p + P).  Token i of sequence b stands at positions[b, i] (int32 [B, N]), or at first[b] + i
    (int32 [B]), or at i; beyond the table the nearest row counts.  backward: the gradient with respect to the rows of a gradient x
    with respect to the turned rows; that of a call on an x that requires a gradient is recorded, and made so (out is for calls without
    one; table, positions and first have none).  out may be x."""
    if (x.requires_grad or table.requires_grad or (out is not None and out.requires_grad)) and torch.is_grad_enabled():
        if out is not None:
            raise ValueError("out: not for a call that a gradient is recorded of")
        if table.requires_grad:
            raise ValueError("table: a gradient with respect to it is not made (detach it)")
        return _Turn.apply(x, table, positions, first, half, backward)
    return _rope(x, table, positions, first, half, backward, out)


class _Turn(torch.autograd.Function):
    """rope with its gradient, which is the turn back by the same rows."""

    @staticmethod
    def forward(ctx, x, table, positions, first, half, backward):
        # (copies: a step's lengths, which first often is, move on before its gradient comes)
        ctx.save_for_backward(table, *(None if t is None else t.clone() for t in (positions, first)))
        ctx.half, ctx.back = half, not backward
        return _rope(x, table, positions, first, half, backward, None)

    @staticmethod
    def backward(ctx, g):
        if g.stride(3) != 1 or g.data_ptr() % 16 or any(s * g.element_size() % 16 for s in g.stride()[:3]):
            g = g.clone(memory_format=torch.contiguous_format)
        return rope(g, *ctx.saved_tensors, ctx.half, ctx.back), None, None, None, None, None


def _rope(x, table, positions, first, half, backward, out):
    _all_here(x, table, positions, first, out)
    xs = _rows_of(x, "x")
    n, H, m, d = x.shape
    if positions is not None and first is not None:
        raise ValueError("positions and first both say where tokens stand")
    r = _rotary(table, half, positions, (n, m))
    if out is None:
        out = torch.empty(n, H, m, d, dtype=x.dtype, device=x.device)
        o0, o1, o2 = H * m * d, m * d, d
    else:
        os_ = _rows_of(out, "out", x.dtype, x.shape, True)
        if out.data_ptr() == x.data_ptr():
            _same_strides(xs, os_, x.shape, ("x", "out"))
            os_ = xs
        o0, o1, o2, _ = os_
    st = lib().qvg_rope(r, TYPES[x.dtype], n, H, m, d, x.data_ptr(), xs[0], xs[1], xs[2], None if first is None else _counts(first, (n,), "first"),
                        1 if backward else 0, out.data_ptr(), o0, o1, o2, _stream())
    if st != 0:
        raise QvgError(st, "qvg_rope")
    return out


def alloc_pages(heads, n_pages, page_len, head_dim=128, dtype=torch.bfloat16, device="cuda"):
    """Uninitialised pages of a cache in 16 bits: (k_pages, v_pages), [heads, n_pages, page_len, head_dim] each."""
    pool = torch.empty(2, heads, n_pages, page_len, head_dim, dtype=dtype, device=device)
    return pool[0], pool[1]


def _page_cache(k_pages, v_pages, page_table, kv_len, written=False) -> QvgPageCache:
    shape, table, dtype = k_pages.shape, page_table.shape, k_pages.dtype
    if dtype is not torch.bfloat16 and dtype is not torch.float16:
        raise TypeError("k_pages: pages are bfloat16 or float16")
    ks = _two_rows(k_pages, v_pages, ("k_pages", "v_pages"), dtype, written)
    if len(table) != 2:
        raise ValueError("page_table: need [B, M]")
    n, pages = table
    return QvgPageCache(TYPES[dtype], n, shape[0], shape[3], pages, 0, shape[2], shape[1], _counts(page_table, table, "page_table"),
                        _counts(kv_len, (n,), "kv_len"), k_pages.data_ptr(), v_pages.data_ptr(), ks[0], ks[1], ks[2] if shape[2] > 1 else 0)


def append_pages(k_new, v_new, k_pages, v_pages, page_table, kv_len, n_new=None, k_rope=None, positions=None, half=False,
                 out_len=None) -> torch.Tensor:
    """qvg_append_pages: the new tokens' K and V [B, H, N, d] go behind B sequences in pages k_pages, v_pages [H, P, L, d] (alloc_pages; any
    views with unit stride along d that share their strides, a token's heads side by side among them).  page_table [B, M] int32: the
    sequences' pages, kv_len [B] int32: their tokens so far, n_new [B] int32: how many of the N are there (None: all).
    k_rope [n, P, 2]: K is turned on the way, by the row of its place in the sequence, or of positions [B, N] int32; half as in rope.
    Returns the new lengths [B] int32 (out_len, which may be kv_len, or a new tensor).  Tokens beyond the table, and those of pages
    outside the pool, are left out.  Any d that is a multiple of 8 up to 512; attn_pages reads pages of 64, 96, 128, 192 and 256."""
    _all_here(k_new, v_new, k_pages, v_pages, page_table, kv_len, n_new, k_rope, positions, out_len)
    c = _page_cache(k_pages, v_pages, page_table, kv_len, True)
    ns = _two_rows(k_new, v_new, ("k_new", "v_new"), k_pages.dtype)
    n, H, m, d = k_new.shape
    if n != c.n_seqs or H != c.n_heads or d != c.head_dim:
        raise ValueError(f"k_new: need [{c.n_seqs}, {c.n_heads}, N, {c.head_dim}]")
    r = None
    if k_rope is not None:
        r = _rotary(k_rope, half, positions, (n, m))
    elif positions is not None:
        raise ValueError("positions without k_rope: keys are not turned")
    out_len = torch.empty(n, dtype=torch.int32, device=kv_len.device) if out_len is None else out_len
    st = lib().qvg_append_pages(c, m, k_new.data_ptr(), v_new.data_ptr(), ns[0], ns[1], ns[2], None if n_new is None else _counts(n_new, (n,), "n_new"),
                                r, _counts(out_len, (n,), "out_len"), _stream())
    if st != 0:
        raise QvgError(st, "qvg_append_pages")
    return out_len


@functools.lru_cache(maxsize=256)
def _pages_scratch_bytes(n_seqs, H, d, group, n_new, table_pages, page_len, window, sink) -> int:
    """Bytes of scratch of an attn_pages of these sizes (a function of its arguments alone)."""
    need = C.c_size_t()
    c = QvgPageCache(n_seqs=n_seqs, n_heads=H, head_dim=d, table_pages=table_pages, page_len=page_len, pool_pages=1)
    st = lib().qvg_attn_pages_scratch_bytes(C.byref(c), C.byref(QvgPageStep(group=group, n_new=n_new, window=window, sink=sink)), C.byref(need))
    if st != 0:
        raise QvgError(st, "qvg_attn_pages_scratch_bytes")
    return need.value


def attn_pages_scratch(k_pages, n_seqs, group, n_new, table_pages) -> torch.Tensor:
    """Scratch for an attn_pages of these sizes over the pages k_pages, with a window or without."""
    H, _, L, d = k_pages.shape
    return torch.empty(_pages_scratch_bytes(n_seqs, H, d, group, n_new, table_pages, L, 0, 0), dtype=torch.uint8, device=k_pages.device)


def attn_pages(q, k_pages, v_pages, page_table, kv_len, n_new=None, causal=True, window=None, sink=0, softmax_scale=None, want_lse=False,
               out=None, scratch=None):
    """qvg_attn_pages: attention of the new tokens' queries q [B, H * group, N, d] over their sequences' pages (append_pages; kv_len [B] counts
    the new tokens) -> out like q (and lse fp32 [B, H * group, N]); query head h reads KV head h // group.
    n_new [B] int32: how many of the N there are (None: all); row i of a sequence stands at place kv_len - n_new + i and sees the
    tokens up to its place (causal), or all kv_len, and with a window only the newest `window` of its place and the first `sink` tokens.
    Rows behind n_new, and those that see nothing, are zero with lse -inf.  The result carries no gradient.
    scratch: uint8 tensor of attn_pages_scratch bytes for dividing the call over the chip; without one it is taken from torch's
    allocator (where that has no memory left the call runs undivided, which differs by the order of fp32 sums)."""
    _all_here(q, k_pages, v_pages, page_table, kv_len, n_new, out, scratch)
    c = _page_cache(k_pages, v_pages, page_table, kv_len)
    q0, q1, q2, _ = _rows_of(q, "q", k_pages.dtype)
    n, hq, m, d = q.shape
    H, L, pages = c.n_heads, c.page_len, c.table_pages
    group = hq // H
    if n != c.n_seqs or d != c.head_dim or group < 1 or group * H != hq:
        raise ValueError(f"q: need [{c.n_seqs}, a multiple of {H} heads, N, {c.head_dim}]")
    if window is not None and window < 1:
        raise ValueError("window: a row sees its own place at least (None: no window)")
    device = q.device
    if out is None:
        out = torch.empty(n, hq, m, d, dtype=q.dtype, device=device)
        o0, o1, o2 = hq * m * d, m * d, d
    else:
        o0, o1, o2, _ = _rows_of(out, "out", q.dtype, q.shape, True)
    lse = torch.empty(n, hq, m, dtype=torch.float32, device=device) if want_lse else None
    window, sink = 0 if window is None else min(window, 0x7fffffff), max(min(sink, 0x7fffffff), -1)      # (ctypes keeps the low bits only)
    if scratch is None:
        scratch = _scratch(_pages_scratch_bytes(n, H, d, group, m, pages, L, window, sink), device)
    elif scratch.dtype is not torch.uint8 or not scratch.is_contiguous():
        raise ValueError("scratch: need a contiguous uint8 tensor")
    t = QvgPageStep(group, m, None if n_new is None else _counts(n_new, (n,), "n_new"), q.data_ptr(), q0, q1, q2, 1 if causal else 0,
                    window, sink, 0, out.data_ptr(), o0, o1, o2, None if lse is None else lse.data_ptr())
    at, size = (None, 0) if scratch is None else (scratch.data_ptr(), scratch.numel())
    st = lib().qvg_attn_pages(c, t, d ** -0.5 if softmax_scale is None else softmax_scale, at, size, _stream())
    if st != 0:
        raise QvgError(st, "qvg_attn_pages")
    return (out, lse) if want_lse else out


def kmeans_assign(x, centroids) -> torch.Tensor:
    """qvg_kmeans_assign -> ids [H, N], uint8 (int16 with more than 256 centroids)."""
    sh, st_ = _view3(x, "x")
    H, N, d = x.shape
    centroids = centroids.contiguous()
    p = make_params(H, centroids.shape[-2], 64, 1, 0, head_dim=d)
    ids = torch.empty(H, N, dtype=id_dtype(centroids.shape[-2]), device=x.device)
    need = workspace_bytes(p, ENTRY_KMEANS_ASSIGN, N)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=x.device)
    st = lib().qvg_kmeans_assign(C.byref(p), N, _ptr(x), sh, st_, _ptr(centroids), _ptr(ids), _ptr(ws), need,
                                 _stream())
    if st != 0:
        raise QvgError(st, "qvg_kmeans_assign")
    return ids


def kmeans_update(x, ids, centroids_prev):
    """qvg_kmeans_update -> (centroids bf16 [H, K, d], counts int32 [H, K])."""
    sh, st_ = _view3(x, "x")
    H, N, d = x.shape
    centroids_prev = centroids_prev.contiguous()
    K = centroids_prev.shape[-2]
    _check(ids, id_dtype(K), "ids")
    p = make_params(H, K, 64, 1, 0, head_dim=d)
    cent = torch.empty(H, K, d, dtype=torch.bfloat16, device=x.device)
    counts = torch.empty(H, K, dtype=torch.int32, device=x.device)
    need = workspace_bytes(p, ENTRY_KMEANS_UPDATE, N)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=x.device)
    st = lib().qvg_kmeans_update(C.byref(p), N, _ptr(x), sh, st_, _ptr(ids.contiguous()),
                                 _ptr(centroids_prev), _ptr(cent), _ptr(counts), _ptr(ws), need, _stream())
    if st != 0:
        raise QvgError(st, "qvg_kmeans_update")
    return cent, counts


class StreamingCache:
    """The compressed K and V cache of one layer during a chunk-by-chunk rollout (paper Sec. 3.1,
    4.3): allocated once for `capacity_tokens`, filled by `append`, read by `attend` / `decode`.
    K heads and V heads are stacked as 2 * heads independent units so that one library call
    encodes both.  Every chunk but the last appended one must be full (chunk_len tokens).
    Argument marshalling only: every step runs in the library's kernels.

    A chunk's k-means starts from the previous chunk's centroids (Sec. 4.3: centroid caching) and
    runs `warm_iters` Lloyd iterations; the first chunk starts from `init` ([2 * heads, K, d], or
    [2 * heads, S, K, d] with S smoothing stages) and runs `cold_iters`."""

    def __init__(self, heads, capacity_tokens, chunk_len, n_clusters, group_size, n_stages, head_dim=128,
                 device="cuda", n_smooth=1, bits=2, scale_format=SCALE_F16, warm_iters=3, cold_iters=10):
        self.heads, self.chunk_len = heads, chunk_len
        self.group_size, self.n_stages = group_size, n_stages
        self.warm_iters, self.cold_iters = warm_iters, cold_iters
        self.cache = alloc_cache(2 * heads, capacity_tokens, chunk_len, n_clusters, group_size, n_stages, head_dim,
                                 device, n_smooth=n_smooth, bits=bits, scale_format=scale_format)
        self.n_tokens = 0
        p = make_params(2 * heads, n_clusters, group_size, n_stages, max(warm_iters, cold_iters), head_dim=head_dim,
                        bits=bits, n_smooth_stages=n_smooth, scale_format=scale_format)
        need = workspace_bytes(p, ENTRY_ENCODE, chunk_len)
        self._ws = torch.empty(max(need, 16), dtype=torch.uint8, device=device)

    @property
    def capacity(self) -> int:
        return self.cache.ids.shape[1]

    def _side(self, lo, hi) -> Encoded:
        c = self.cache
        return Encoded(c.centroids[lo:hi], c.ids[lo:hi], c.codes[lo:hi], c.scales[lo:hi], c.chunk_len, c.n_smooth)

    @property
    def k(self) -> Encoded:
        return self._side(0, self.heads)

    @property
    def v(self) -> Encoded:
        return self._side(self.heads, 2 * self.heads)

    def append(self, kv_chunk, init=None, iters=None) -> int:
        """Encode one chunk, kv_chunk [2 * heads, n, d] bf16 (K heads first), n <= chunk_len, at the
        end of the cache.  Returns the chunk's index."""
        if self.n_tokens % self.chunk_len != 0:
            raise ValueError("the previous chunk was not full: nothing can be appended after it")
        n = kv_chunk.shape[1]
        if n < 1 or n > self.chunk_len or self.n_tokens + n > self.capacity:
            raise ValueError("chunk does not fit")
        c = self.n_tokens // self.chunk_len
        if c > 0 and init is None:
            init = self.cache.centroids[:, c - 1]
            iters = self.warm_iters if iters is None else iters
        elif init is None:
            raise ValueError("the first chunk needs start centroids")
        else:
            iters = (self.cold_iters if c == 0 else self.warm_iters) if iters is None else iters
        encode_chunk(kv_chunk, init, self.group_size, self.n_stages, iters, cache=self.cache, chunk_index=c,
                     workspace=self._ws)
        self.n_tokens += n
        return c

    def attend(self, q, k_rope=None, softmax_scale=None, want_lse=False, out=None, workspace=None):
        """Attention of q [heads, n_q, d] over the tokens appended so far (decode fused in)."""
        if self.n_tokens == 0:
            raise ValueError("the cache is empty")
        # the two halves of the cache by address: views of both sides (self.k, self.v) cost more than the
        # smallest attention's launches
        c = self.cache
        h = self.heads
        kp = (c.centroids.data_ptr(), c.ids.data_ptr(), c.codes.data_ptr(), c.scales.data_ptr())
        vp = (kp[0] + h * c.centroids.stride(0) * 2, kp[1] + h * c.ids.stride(0) * c.ids.element_size(),
              kp[2] + h * c.codes.stride(0), kp[3] + h * c.scales.stride(0) * c.scales.element_size())
        return _attn(q, c, kp, vp, softmax_scale, want_lse, out, self.n_tokens, k_rope, None,
                     False, workspace)

    def decode(self, out=None, first_chunk=0, n_tokens=None) -> torch.Tensor:
        """bf16 [2 * heads, n, d] of the tokens appended so far, from chunk `first_chunk` on."""
        first = first_chunk * self.chunk_len
        n = self.n_tokens - first if n_tokens is None else n_tokens
        if first + n > self.n_tokens:
            raise ValueError("range beyond the tokens appended so far")
        return decode(self.cache, out=out, n_tokens=n, first_token=first)

    def stored_bytes(self) -> int:
        """Bytes the appended tokens occupy (codes, scales, ids and the chunks' tables)."""
        c = self.cache
        per_tok = c.codes.shape[2] * c.codes.shape[3] + c.scales.shape[2] * c.scales.shape[3] * c.scales.element_size() \
            + c.n_smooth * c.ids.element_size()
        chunks = -(-self.n_tokens // self.chunk_len)
        table = c.n_smooth * c.centroids.shape[-2] * c.centroids.shape[-1] * 2
        return 2 * self.heads * (self.n_tokens * per_tok + chunks * table)


class PagedCache:
    """The compressed K and V caches of one layer of up to `max_seqs` sequences over one pool of `n_pages` pages of page_len
    tokens (K heads, then V heads, as 2 * heads units).  A sequence's tokens go into a bf16 tail first and, whenever page_len
    of them are there, through the encoder into a page of their own (k-means started from the sequence's page before, Sec. 4.3;
    from `init` [2 * heads, K, d] or [2 * heads, S, K, d] for its first).  Pages never change once they are written, so `fork`
    shares them and copies the tail only; `close` gives back those that no other sequence holds; `compact` moves the used ones
    to the pool's front.  A step attends with a row of new tokens for every place 0 .. max_seqs - 1 (places that are not open
    have none) and then keeps those that were accepted.
    Keys are stored as they are attended to, or with pre_rope=True as they were before the rotary embedding (the codec's own
    scheme): pages then hold them so and attend rotates them by their place (k_rope), while the tail holds both forms, the one
    for the encoder and the one that is attended to.  append and keep take the stored form, and the rotated one beside it.
    Argument marshalling and page numbers only: every step runs in the library's kernels."""

    def __init__(self, heads, max_seqs, n_pages, page_len, max_pages, max_new, n_clusters, group_size, n_stages, init, head_dim=128,
                 device="cuda", n_smooth=1, bits=2, scale_format=SCALE_F16, warm_iters=3, cold_iters=10, pre_rope=False):
        if scale_format == SCALE_F16 and page_len * n_stages * (head_dim // group_size) % 8:
            raise ValueError("page_len: a page's binary16 scales must fill multiples of 16 bytes (8 tokens always do)")
        self.heads, self.page_len, self.max_new, self.pre_rope = heads, page_len, max_new, pre_rope
        self.group_size, self.n_stages = group_size, n_stages
        self.init, self.warm_iters, self.cold_iters = init, warm_iters, cold_iters
        self.pool = alloc_cache(2 * heads, n_pages * page_len, page_len, n_clusters, group_size, n_stages, head_dim, device,
                                n_smooth=n_smooth, bits=bits, scale_format=scale_format)
        # (units: K heads as stored, V heads, and with pre_rope the K heads as attended to)
        self.tail = torch.empty(max_seqs, (3 if pre_rope else 2) * heads, page_len + max_new, head_dim, dtype=torch.bfloat16, device=device)
        self.table = torch.zeros(max_seqs, max_pages, dtype=torch.int32, device=device)
        self.kv_len = torch.zeros(max_seqs, dtype=torch.int32, device=device)
        self.tail_len = torch.zeros(max_seqs, dtype=torch.int32, device=device)
        self.pages = [None] * max_seqs                 # a sequence's pages in order; None: the place is not open
        self.tails = [0] * max_seqs                    # tokens in the tail, as on the device
        self.holders = [0] * n_pages                   # sequences that hold a page
        p = make_params(2 * heads, n_clusters, group_size, n_stages, max(warm_iters, cold_iters), head_dim=head_dim, bits=bits,
                        n_smooth_stages=n_smooth, scale_format=scale_format)
        self._ws = torch.empty(max(workspace_bytes(p, ENTRY_ENCODE, page_len), 16), dtype=torch.uint8, device=device)

    def free_pages(self) -> int:
        return self.holders.count(0)

    def length(self, seq) -> int:
        return len(self._open(seq)) * self.page_len + self.tails[seq]

    def _open(self, seq):
        if not 0 <= seq < len(self.pages) or self.pages[seq] is None:
            raise ValueError(f"sequence {seq} is not open")
        return self.pages[seq]

    def _tails(self):
        """The tails' K as attended to, and V."""
        h = self.heads
        return self.tail[:, 2 * h:] if self.pre_rope else self.tail[:, :h], self.tail[:, h:2 * h]

    def _check_rotated(self, k_rotated):
        if (k_rotated is not None) != self.pre_rope:
            raise ValueError("k_rotated: needed by a cache of pre_rope keys, and by no other")

    def _place(self):
        if None not in self.pages:
            raise ValueError("all places are taken")
        return self.pages.index(None)

    def _tell(self, seq):
        """The device's copy of a sequence's pages and lengths."""
        pages = self.pages[seq] or []
        if pages:
            self.table[seq, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
        self.kv_len[seq], self.tail_len[seq] = len(pages) * self.page_len, self.tails[seq]

    def open(self) -> int:
        """A new, empty sequence; returns its place."""
        seq = self._place()
        self.pages[seq], self.tails[seq] = [], 0
        self._tell(seq)
        return seq

    def fork(self, seq) -> int:
        """A copy of a sequence: its pages are shared, its tail is copied."""
        pages, to = self._open(seq), self._place()
        for page in pages:
            self.holders[page] += 1
        self.pages[to], self.tails[to] = list(pages), self.tails[seq]
        self.tail[to, :, :self.tails[seq]].copy_(self.tail[seq, :, :self.tails[seq]])
        self._tell(to)
        return to

    def close(self, seq):
        """End a sequence; pages that no other one holds are free again."""
        for page in self._open(seq):
            self.holders[page] -= 1
        self.pages[seq], self.tails[seq] = None, 0
        self._tell(seq)

    def _need(self, tokens_of):
        """Refuses what the pool or a table has no room for, before anything is changed: {sequence: tokens to come}."""
        more = 0
        for seq, n in tokens_of.items():
            new = (self.tails[seq] + n) // self.page_len
            if len(self._open(seq)) + new > self.table.shape[1]:
                raise ValueError(f"sequence {seq} would have more than {self.table.shape[1]} pages")
            more += new
        if more > self.free_pages():
            raise ValueError(f"{more} pages are needed, {self.free_pages()} are free")

    def _encode(self, seq, x):
        """One full page of a sequence, x [2 * heads, page_len, d]."""
        pages, page = self.pages[seq], self.holders.index(0)
        init = self.pool.centroids[:, pages[-1]] if pages else self.init
        encode_chunk(x, init, self.group_size, self.n_stages, self.warm_iters if pages else self.cold_iters, cache=self.pool,
                     chunk_index=page, workspace=self._ws)
        self.holders[page] = 1
        pages.append(page)

    def _seal(self, seq):
        """Full pages leave the tail.  Those that an encoder's error kept there wait for the next call."""
        L, n = self.page_len, self.tails[seq]
        full = 0
        try:
            while n - full >= L:
                self._encode(seq, self.tail[seq, :2 * self.heads, full:full + L])
                full += L
        finally:
            if full:
                if n > full:
                    self.tail[seq, :, :n - full].copy_(self.tail[seq, :, full:n].clone())
                self.tails[seq] = n - full
                self._tell(seq)

    def append(self, seq, kv, k_rotated=None, k_rope=None):
        """Tokens that are there already (a prompt), kv [2 * heads, n, d] bf16 (K heads first), behind the sequence.  pre_rope: kv
        holds the keys before the rotary embedding, k_rotated [heads, n, d] bf16 the same ones rotated by their places; or k_rope
        [n, d/2, 2] is the table that attend is given, with a row for every place of the sequence and the new tokens, and they are
        rotated here (rope)."""
        units, d = 2 * self.heads, self.tail.shape[3]
        if kv.dim() != 3 or kv.shape[0] != units or kv.shape[2] != d:
            raise ValueError(f"kv: need [{units}, n, {d}]")
        _check(kv, torch.bfloat16, "kv")
        if k_rope is not None:
            if k_rotated is not None:
                raise ValueError("k_rotated and k_rope both give the rotated keys")
            if not self.pre_rope:
                raise ValueError("k_rope: needed by a cache of pre_rope keys, and by no other")
            if k_rope.dim() != 3 or k_rope.shape[1] != d // 2:
                raise ValueError(f"k_rope: need [n, {d // 2}, 2]")
            end = self.length(seq) + kv.shape[1]
            if k_rope.shape[0] < end:                  # (beyond a table its last row would count: keys of another place)
                raise ValueError(f"k_rope: need the rows of {end} places, got {k_rope.shape[0]}")
            self._need({seq: kv.shape[1]})
            k_rotated = rope(kv[None, :self.heads], k_rope, first=self.kv_len[seq:seq + 1] + self.tail_len[seq:seq + 1])[0]
        self._check_rotated(k_rotated)
        if k_rotated is not None:
            if k_rotated.shape != (self.heads, kv.shape[1], d):
                raise ValueError(f"k_rotated: need [{self.heads}, {kv.shape[1]}, {d}]")
            _check(k_rotated, torch.bfloat16, "k_rotated")
        _here(self.tail, self.init, kv, k_rotated)
        n, L = kv.shape[1], self.page_len
        self._need({seq: n})
        try:
            self._seal(seq)
            at = 0
            if self.tails[seq] == 0:                   # whole pages need no way through the tail
                while n - at >= L:
                    self._encode(seq, kv[:, at:at + L])
                    at += L
            while at < n:
                m = min(n - at, L - self.tails[seq])
                rows = self.tail[seq, :, self.tails[seq]:self.tails[seq] + m]
                rows[:units].copy_(kv[:, at:at + m])
                if k_rotated is not None:
                    rows[units:].copy_(k_rotated[:, at:at + m])
                self.tails[seq] += m
                at += m
                self._seal(seq)
        finally:                                       # (after an error: the tokens that length counts are there)
            self._tell(seq)

    def attend(self, q, k_new, v_new, n_nodes=None, mask=None, k_rope=None, softmax_scale=None, want_lse=False, out=None,
               scratch=None):
        """attn_tree of q [max_seqs, heads * group, N, d] over the sequences and the new tokens k_new, v_new
        [max_seqs, heads, N, d] (k_new as attended to).  n_nodes [max_seqs] int32: a place's new tokens (None: all N; pass 0 for
        places that are not open, or ignore their rows).  k_rope [n, d/2, 2] float16: the rotary table of a cache of pre_rope
        keys; no other takes one (its pages hold keys that are rotated already, or none is)."""
        if (k_rope is not None) != self.pre_rope:
            raise ValueError("k_rope: needed by a cache of pre_rope keys, and by no other")
        c, h = self.pool, self.heads
        kp = (c.centroids.data_ptr(), c.ids.data_ptr(), c.codes.data_ptr(), c.scales.data_ptr())
        vp = (kp[0] + h * c.centroids.stride(0) * 2, kp[1] + h * c.ids.stride(0) * c.ids.element_size(),
              kp[2] + h * c.codes.stride(0), kp[3] + h * c.scales.stride(0) * c.scales.element_size())
        return _attn_tree(q, c, kp, vp, h, self.table, self.kv_len, k_new, v_new, *self._tails(), self.tail_len, n_nodes, mask,
                          softmax_scale, k_rope, want_lse, out, scratch)

    def keep(self, k_new, v_new, path, n_keep, k_rotated=None):
        """Accepted new tokens become part of the sequences: path [max_seqs, M] int32 on the device (M <= max_new), the indices of
        the kept ones in order; n_keep: how many of each, max_seqs Python integers.  pre_rope: k_new holds the keys before the
        rotary embedding, k_rotated [max_seqs, heads, N, d] those that attend was given."""
        self._check_rotated(k_rotated)
        n_keep = [int(n) for n in n_keep]
        if len(n_keep) != len(self.pages) or path.shape[1] > self.max_new or any(not 0 <= n <= path.shape[1] for n in n_keep):
            raise ValueError(f"n_keep: need {len(self.pages)} counts of at most {min(path.shape[1], self.max_new)} tokens")
        kept = {s: n for s, n in enumerate(n_keep) if n}
        self._need(kept)
        for seq in kept:                               # (room for max_new behind less than a page)
            self._seal(seq)
        h = self.heads
        count, (tail_k, tail_v) = torch.tensor(n_keep, dtype=torch.int32, device=path.device), self._tails()
        if k_rotated is not None:                      # (and V, which comes again with the same values)
            keep_nodes(k_rotated, v_new, path, count, tail_k, tail_v, self.tail_len)
        keep_nodes(k_new, v_new, path, count, self.tail[:, :h], tail_v, self.tail_len, out_len=self.tail_len)
        for seq, n in kept.items():
            self.tails[seq] += n
        for seq in kept:
            self._seal(seq)

    def compact(self) -> int:
        """Moves the used pages to the pool's front and returns how many there are."""
        used = [i for i, n in enumerate(self.holders) if n]
        holes = [i for i in range(len(used)) if not self.holders[i]]
        moved = dict(zip([i for i in used if i >= len(used)], holes))
        if moved:
            copy_pages(self.pool, list(moved), list(moved.values()))
            for a, b in moved.items():
                self.holders[a], self.holders[b] = 0, self.holders[a]
            for seq, pages in enumerate(self.pages):
                if pages and any(p in moved for p in pages):
                    self.pages[seq] = [moved.get(p, p) for p in pages]
                    self._tell(seq)
        return len(used)

    def gather(self, seq, into: Encoded | None = None) -> Encoded:
        """A sequence's pages one behind the other in a cache of their own (`into`, or a new one), as decode and attn_decode
        read it.  Units: K heads, then V heads."""
        pages, c = self._open(seq), self.pool
        if not pages:
            raise ValueError("the sequence has no full page yet")
        if into is None:
            d = c.centroids.shape[-1]
            into = alloc_cache(2 * self.heads, len(pages) * self.page_len, self.page_len, c.centroids.shape[-2], self.group_size,
                               self.n_stages, d, c.ids.device, n_smooth=c.n_smooth, bits=c.bits, scale_format=c.scale_format)
        return copy_pages(c, pages, list(range(len(pages))), into=into)
