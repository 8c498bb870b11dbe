"""ctypes binding of the attention half of a decoded token: rotary positions, the append to a paged cache and the
attention that reads it.  Argument marshalling only, as in :mod:`.binding`; functions have the names and meanings of
their C counterparts in ``include/moesys.h``.

Tensors of tokens are ``[tokens, heads, head_dim]`` CUDA tensors whose last dimension is contiguous; the other two may
have any strides (the queries inside the output of a fused projection).
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import torch

from . import binding as B

_MAX_AXES = 3
_MAX_INT = 2 ** 31 - 1


class _HeadRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class _RotarySpec(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("n_axes", C.c_int32),
                ("axis_pairs", C.c_int32 * _MAX_AXES), ("freqs", C.c_void_p)]


class _Cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_table", C.c_void_p), ("n_pages", C.c_int64),
                ("page_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64),
                ("page_size", C.c_int32), ("n_seqs", C.c_int32), ("table_width", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class _Options(C.Structure):
    _fields_ = [("scale", C.c_float), ("softcap", C.c_float), ("window", C.c_int32), ("slopes", C.c_void_p)]


_DTYPES = {torch.float32: B.MOE_F32, torch.bfloat16: B.MOE_BF16}
_lib = None


def lib() -> C.CDLL:
    """The library with this module's argument types set."""
    global _lib
    if _lib is None:
        L = B.lib()
        vp, rows = C.c_void_p, C.POINTER(_HeadRows)
        L.moe_kv_cache_check.argtypes = [C.POINTER(_Cache)]
        L.moe_rotary.argtypes = [C.POINTER(_RotarySpec), C.c_int32, C.c_int32, C.c_int32, rows, vp, rows, C.c_int32, vp]
        L.moe_kv_append.argtypes = [C.POINTER(_Cache), C.c_int32, rows, rows, vp, vp, C.POINTER(_RotarySpec), vp, C.c_int32, rows, rows, vp]
        L.moe_attention_decode_workspace_bytes.restype = C.c_size_t
        L.moe_attention_decode_workspace_bytes.argtypes = [C.POINTER(_Cache), C.c_int32]
        L.moe_attention_decode.argtypes = [C.POINTER(_Cache), C.c_int32, rows, vp, C.POINTER(_Options), rows, vp, vp, C.c_size_t, vp]
        _lib = L
    return _lib


def _int32(n: int, what: str) -> int:
    """A number that the library takes as int32 (ctypes would cut it down to 32 bits)."""
    if not -_MAX_INT - 1 <= n <= _MAX_INT:
        raise ValueError(f"{what}={n} is beyond int32")
    return n


def _options(scale: float, softcap: float, window: int, slopes: Optional[int]) -> _Options:
    if not -1 <= window <= _MAX_INT:
        window = -1 if window < 0 else _MAX_INT  # (no sequence is longer)
    return _Options(scale, softcap, window, slopes)


def _dtype(t) -> int:
    if t.dtype not in _DTYPES:
        raise ValueError(f"{t.dtype} tensors: float32 and bfloat16 are supported")
    return _DTYPES[t.dtype]


def _rows(t, what: str, shape, dtype, device: int) -> _HeadRows:
    """[tokens, heads, head_dim] as the library takes it, checked against what the call says it holds."""
    if t.shape != shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, the call needs {shape}")
    if t.dtype is not dtype:
        raise ValueError(f"{what} is {t.dtype}, the call needs {dtype}")
    if t.get_device() != device:
        _wrong_device(what, t, device)
    token, head, element = t.stride()
    if element != 1 and shape[2] > 1:
        raise ValueError(f"{what}: the elements of a head must be contiguous")
    return _HeadRows(t.data_ptr(), token, head)


def _vector(t, what: str, dtype, shape, device: int) -> Optional[int]:
    """The address of a contiguous tensor of a shape and dtype."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{what} is a {t.dtype} tensor of shape {tuple(t.shape)}, the call needs a contiguous {dtype} one of shape {shape}")
    if t.get_device() != device:
        _wrong_device(what, t, device)
    return t.data_ptr()


def _wrong_device(what: str, t, device: int) -> None:
    raise ValueError(f"{what} is on {t.device}: device tensors are needed" + (f", here on CUDA device {device}" if device >= 0 else ""))


def _device(t, what: str) -> int:
    device = t.get_device()
    if device < 0:
        _wrong_device(what, t, device)
    return device


def _stream(stream, device: int) -> Optional[int]:
    """The given stream, or the device's current one; the raw handle spares a decoded token's calls the 2.7 us that building
    torch's stream object takes, as much as all their other checks together.  A default stream has no handle of its own: the
    library would launch on the current device, whatever device the tensors are on."""
    handle = torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream
    if stream is not None and stream.device_index != device:
        raise ValueError(f"a stream of CUDA device {stream.device_index} for tensors on device {device}")
    if not handle and torch._C._cuda_getDevice() != device:
        raise ValueError(f"tensors on CUDA device {device}, whose default stream can only be used while it is the current device")
    return handle or None


class Rotary:
    """Rotary positions of a head (moe_rotary_spec): ``freqs`` is a float64 CUDA tensor of rot_dim/2 radians per position,
    ``axis_pairs`` how many of the pairs belong to each axis, in order (default: all to one)."""

    def __init__(self, head_dim: int, freqs, axis_pairs: Optional[Sequence[int]] = None, interleaved: bool = False):
        if freqs.dtype != torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous():
            raise ValueError("freqs must be a contiguous float64 vector")
        self.device = _device(freqs, "freqs")
        pairs = [freqs.numel()] if axis_pairs is None else [_int32(int(n), "axis_pairs") for n in axis_pairs]
        if not 1 <= len(pairs) <= _MAX_AXES:
            raise ValueError(f"{len(pairs)} axes: 1 to {_MAX_AXES} are supported")
        self.freqs, self.head_dim, self.n_axes = freqs, head_dim, len(pairs)
        self.c = _RotarySpec(_int32(head_dim, "head_dim"), _int32(2 * freqs.numel(), "rot_dim"), int(bool(interleaved)), len(pairs),
                             (C.c_int32 * _MAX_AXES)(*(pairs + [0] * (_MAX_AXES - len(pairs)))), freqs.data_ptr())


def rotary_freqs(rot_dim: int, base: float = 10000.0, device="cuda"):
    """The usual geometric series base^(-2i/rot_dim), i < rot_dim/2, in float64."""
    i = torch.arange(rot_dim // 2, dtype=torch.float64)
    return (base ** (-2.0 * i / rot_dim)).to(device)


class KVCache:
    """A paged cache of keys and values (moe_kv_cache): ``k`` and ``v`` are pools of pages, [pages, page_size, heads, head_dim]
    (``token_major``) or [pages, heads, page_size, head_dim] (``head_major``), of one dtype and the same strides (they may be
    halves of one tensor); ``page_table`` is int32 [sequences, width].  Keeps the tensors, and reads their contents anew in
    every call."""

    def __init__(self, k, v, page_table, layout: str = "token_major"):
        if layout not in ("token_major", "head_major"):
            raise ValueError(f"layout {layout!r}: token_major or head_major")
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.stride() != v.stride():
            raise ValueError("k and v must be 4-dimensional pools of one shape, dtype and strides")
        if k.stride(3) != 1:
            raise ValueError("the elements of a head must be contiguous")
        if page_table.dtype != torch.int32 or page_table.dim() != 2 or not page_table.is_contiguous():
            raise ValueError("page_table must be a contiguous int32 matrix")
        self.device = _device(k, "k")
        for t, what in ((v, "v"), (page_table, "page_table")):
            if t.get_device() != self.device:
                _wrong_device(what, t, self.device)
        self.k, self.v, self.page_table, self.layout = k, v, page_table, layout
        tok, head = (1, 2) if layout == "token_major" else (2, 1)
        self.page_size, self.n_kv_heads, self.head_dim = k.shape[tok], k.shape[head], k.shape[3]
        self.n_seqs, self.dtype = page_table.shape[0], k.dtype
        for n in tuple(k.shape[1:]) + tuple(page_table.shape):
            _int32(n, "a dimension of the cache")
        self.scale = self.head_dim ** -0.5
        self.c = _Cache(k.data_ptr() or None, v.data_ptr() or None, page_table.data_ptr() or None, k.shape[0], k.stride(0), k.stride(tok),
                        k.stride(head), self.page_size, page_table.shape[0], page_table.shape[1], self.n_kv_heads, self.head_dim, _dtype(k))
        B._check(lib().moe_kv_cache_check(C.byref(self.c)), "moe_kv_cache_check")


def moe_rotary(rotary: Rotary, x, positions, out, inverse: bool = False, stream=None):
    """out <- x [T, heads, head_dim] rotated by positions [axes, T] (int32; [T] for one axis); ``inverse``: back, or the gradient."""
    shape, dtype, device = tuple(x.shape), x.dtype, rotary.device
    T, H, D = shape
    if T > _MAX_INT or H > _MAX_INT:
        _int32(max(T, H), "tokens or heads")
    if D != rotary.head_dim:
        raise ValueError(f"x has heads of {D}, the rotary positions are for {rotary.head_dim}")
    st = lib().moe_rotary(rotary.c, _dtype(x), T, H, _rows(x, "x", shape, dtype, device), _positions(rotary, positions, T, device),
                          _rows(out, "out", shape, dtype, device), 1 if inverse else 0, _stream(stream, device))
    if st:
        B._check(st, "moe_rotary")


def _positions(rotary: Rotary, positions, T: int, device: int) -> int:
    shape = (T,) if positions.dim() == 1 and rotary.n_axes == 1 else (rotary.n_axes, T)
    return _vector(positions, "positions", torch.int32, shape, device)


def moe_kv_append(cache: KVCache, k, v, cache_pos, token_seq=None, rotary: Optional[Rotary] = None, positions=None, q=None, q_out=None,
                  stream=None):
    """Keys and values [T, kv_heads, head_dim] of new tokens into their places of the cache, keys rotated; queries
    [T, heads, head_dim] rotated into q_out."""
    T, D, dtype, device = k.shape[0], cache.head_dim, cache.dtype, cache.device
    if T > _MAX_INT:
        _int32(T, "tokens")
    shape, per_token = (T, cache.n_kv_heads, D), (T,)
    spec = pos = q_rows = q_out_rows = None
    heads = 0
    if rotary is not None:
        if rotary.device != device:
            raise ValueError(f"rotary positions of CUDA device {rotary.device}, a cache on {device}")
        spec = rotary.c
        if positions is not None:
            pos = _positions(rotary, positions, T, device)
    elif positions is not None:
        raise ValueError("positions without rotary")
    if q is not None:
        if q_out is None:
            raise ValueError("q without q_out")
        heads = q.shape[1]
        if heads > _MAX_INT:
            _int32(heads, "heads")
        q_shape = (T, heads, D)
        q_rows, q_out_rows = _rows(q, "q", q_shape, dtype, device), _rows(q_out, "q_out", q_shape, dtype, device)
    st = lib().moe_kv_append(cache.c, T, _rows(k, "k", shape, dtype, device), _rows(v, "v", shape, dtype, device),
                             _vector(token_seq, "token_seq", torch.int32, per_token, device), _vector(cache_pos, "cache_pos", torch.int32, per_token, device),
                             spec, pos, heads, q_rows, q_out_rows, _stream(stream, device))
    if st:
        B._check(st, "moe_kv_append")


def moe_attention_decode_workspace_bytes(cache: KVCache, n_q_heads: int) -> int:
    n = lib().moe_attention_decode_workspace_bytes(cache.c, _int32(n_q_heads, "n_q_heads"))
    if n == 0:
        raise B.MoEError(1, "moe_attention_decode_workspace_bytes", lib().moe_last_error().decode())
    return n


def moe_attention_decode(cache: KVCache, q, seq_lens, out, ws, scale: Optional[float] = None, softcap: float = 0.0, window: int = 0,
                         slopes=None, lse=None, stream=None):
    """Attention of one new token per sequence: q, out [sequences, heads, head_dim], seq_lens int32 [sequences] (the new token
    counted), slopes float32 [heads] (optional), lse float32 [sequences, heads] (optional output)."""
    S, H, dtype, device = cache.n_seqs, q.shape[1], cache.dtype, cache.device
    if H > _MAX_INT:
        _int32(H, "heads")
    shape = (S, H, cache.head_dim)
    if not ws.is_contiguous() or ws.get_device() != device:
        raise ValueError("the workspace must be contiguous and on the cache's device")
    options = _options(cache.scale if scale is None else scale, softcap, window, _vector(slopes, "slopes", torch.float32, (H,), device))
    st = lib().moe_attention_decode(cache.c, H, _rows(q, "q", shape, dtype, device), _vector(seq_lens, "seq_lens", torch.int32, (S,), device), options,
                                    _rows(out, "out", shape, dtype, device), _vector(lse, "lse", torch.float32, (S, H), device),
                                    ws.data_ptr(), ws.nbytes, _stream(stream, device))
    if st:
        B._check(st, "moe_attention_decode")
