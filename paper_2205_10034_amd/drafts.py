"""ctypes binding of a step of drafted tokens: attention for a tree of them over a paged cache, the places of the accepted
ones, and the cache's pages.  Argument marshalling only, as in :mod:`.attention`; functions have the names and meanings of
their C counterparts in ``include/moesys.h``.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from . import attention as A
from . import binding as B


class _Options(C.Structure):
    _fields_ = [("scale", C.c_float), ("softcap", C.c_float), ("window", C.c_int32), ("sinks", C.c_int32), ("slopes", C.c_void_p)]


_lib = None


def lib() -> C.CDLL:
    """The library with this module's argument types set."""
    global _lib
    if _lib is None:
        L = A.lib()
        vp, i32, cache, rows = C.c_void_p, C.c_int32, C.POINTER(A._Cache), C.POINTER(A._HeadRows)
        L.moe_attention_tree_workspace_bytes.restype = C.c_size_t
        L.moe_attention_tree_workspace_bytes.argtypes = [cache, i32, i32]
        L.moe_attention_tree.argtypes = [cache, i32, i32, i32, rows, vp, vp, vp, C.POINTER(_Options), rows, vp, vp, C.c_size_t, vp]
        L.moe_kv_compact.argtypes = [cache, vp, i32, vp, vp, vp]
        L.moe_kv_release.argtypes = [cache, vp, vp, vp]
        L.moe_kv_pages_workspace_bytes.restype = C.c_size_t
        L.moe_kv_pages_workspace_bytes.argtypes = [cache]
        L.moe_kv_fork.argtypes = [cache, vp, i32, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.moe_kv_reserve.argtypes = [cache, vp, vp, i32, vp, vp, C.c_size_t, vp]
        _lib = L
    return _lib


def _count(n: int) -> int:
    """A window or a number of sinks: no sequence is longer than int32."""
    return n if -1 <= n <= A._MAX_INT else -1 if n < 0 else A._MAX_INT


def _ws(ws, device: int):
    if not ws.is_contiguous() or ws.get_device() != device:
        raise ValueError("the workspace must be contiguous and on the cache's device")
    return ws.data_ptr(), ws.nbytes


def moe_attention_tree_workspace_bytes(cache: A.KVCache, n_q_heads: int, max_new: int) -> int:
    n = lib().moe_attention_tree_workspace_bytes(cache.c, A._int32(n_q_heads, "n_q_heads"), A._int32(max_new, "max_new"))
    if n == 0:
        raise B.MoEError(1, "moe_attention_tree_workspace_bytes", lib().moe_last_error().decode())
    return n


def moe_attention_tree(cache: A.KVCache, q, token_first, seq_lens, out, ws, max_new: int, visible=None, scale: Optional[float] = None,
                       softcap: float = 0.0, window: int = 0, sinks: int = 0, slopes=None, lse=None, stream=None):
    """Attention of each sequence's new tokens: q, out [T, heads, head_dim], token_first int32 [sequences + 1], seq_lens int32
    [sequences] (the new tokens counted), max_new the most new tokens of a sequence in this step, visible int64 [T] (bit j: the sequence's j-th new token; None: a chain), slopes
    float32 [heads] (optional), lse float32 [T, heads] (optional output)."""
    S, dtype, device = cache.n_seqs, cache.dtype, cache.device
    T, H = q.shape[0], q.shape[1]
    if H > A._MAX_INT or T > A._MAX_INT:
        A._int32(max(H, T), "tokens or heads")
    shape = (T, H, cache.head_dim)
    ws_at, ws_bytes = _ws(ws, device)
    options = _Options(cache.scale if scale is None else scale, softcap, _count(window), _count(sinks), A._vector(slopes, "slopes", torch.float32, (H,), device))
    st = lib().moe_attention_tree(cache.c, H, T, A._int32(max_new, "max_new"), A._rows(q, "q", shape, dtype, device),
                                  A._vector(token_first, "token_first", torch.int32, (S + 1,), device), A._vector(seq_lens, "seq_lens", torch.int32, (S,), device),
                                  A._vector(visible, "visible", torch.int64, (T,), device), options, A._rows(out, "out", shape, dtype, device),
                                  A._vector(lse, "lse", torch.float32, (T, H), device), ws_at, ws_bytes, A._stream(stream, device))
    if st:
        B._check(st, "moe_attention_tree")


def moe_kv_compact(cache: A.KVCache, base, keep, new_lens=None, stream=None):
    """The accepted drafts keep [sequences, width] (int32, a negative one ends a row) of every sequence move up to base [sequences]."""
    S, device = cache.n_seqs, cache.device
    if keep.dim() != 2:
        raise ValueError("keep must be a matrix [sequences, width]")
    width = keep.shape[1]
    st = lib().moe_kv_compact(cache.c, A._vector(base, "base", torch.int32, (S,), device), A._int32(width, "width"),
                              A._vector(keep, "keep", torch.int32, (S, width), device), A._vector(new_lens, "new_lens", torch.int32, (S,), device),
                              A._stream(stream, device))
    if st:
        B._check(st, "moe_kv_compact")


def moe_kv_pages_workspace_bytes(cache: A.KVCache) -> int:
    n = lib().moe_kv_pages_workspace_bytes(cache.c)
    if n == 0:
        raise B.MoEError(1, "moe_kv_pages_workspace_bytes", lib().moe_last_error().decode())
    return n


def _refs(cache: A.KVCache, refs):
    return A._vector(refs, "refs", torch.int32, (cache.c.n_pages,), cache.device)


def moe_kv_release(cache: A.KVCache, refs, lens, stream=None):
    """Pages behind the first lens [sequences] places of every sequence are given back; refs int32 [pages]."""
    device = cache.device
    st = lib().moe_kv_release(cache.c, _refs(cache, refs), A._vector(lens, "lens", torch.int32, (cache.n_seqs,), device), A._stream(stream, device))
    if st:
        B._check(st, "moe_kv_release")


def moe_kv_fork(cache: A.KVCache, refs, src, dst, lens, ws, missing=None, stream=None):
    """Sequences dst become others of sequences src (int32 [n] each), sharing their whole pages; lens [sequences] follows."""
    device = cache.device
    if src.dim() != 1:
        raise ValueError("src must be a vector")
    n = src.shape[0]
    ws_at, ws_bytes = _ws(ws, device)
    st = lib().moe_kv_fork(cache.c, _refs(cache, refs), A._int32(n, "n"), A._vector(src, "src", torch.int32, (n,), device),
                           A._vector(dst, "dst", torch.int32, (n,), device), A._vector(lens, "lens", torch.int32, (cache.n_seqs,), device),
                           A._vector(missing, "missing", torch.int32, (1,), device), ws_at, ws_bytes, A._stream(stream, device))
    if st:
        B._check(st, "moe_kv_fork")


def moe_kv_reserve(cache: A.KVCache, refs, lens, ws, more: int = 0, missing=None, stream=None):
    """Every sequence gets the pages that its first lens [sequences] + more places lack."""
    device = cache.device
    ws_at, ws_bytes = _ws(ws, device)
    st = lib().moe_kv_reserve(cache.c, _refs(cache, refs), A._vector(lens, "lens", torch.int32, (cache.n_seqs,), device), A._int32(more, "more"),
                              A._vector(missing, "missing", torch.int32, (1,), device), ws_at, ws_bytes, A._stream(stream, device))
    if st:
        B._check(st, "moe_kv_reserve")
