"""ctypes binding of the log-probabilities of tokens and their gradient.  Argument marshalling only; functions have the
names and meanings of their C counterparts in ``include/moesys.h``."""
from __future__ import annotations

import ctypes as C

import torch

from . import attention as A
from . import binding as B

_lib = None


def lib() -> C.CDLL:
    """The library with this module's argument types set."""
    global _lib
    if _lib is None:
        L = B.lib()
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        L.moe_token_logprobs_workspace_bytes.restype = C.c_size_t
        L.moe_token_logprobs_workspace_bytes.argtypes = [i32, i32, i32]
        L.moe_token_logprobs.argtypes = [i32, i32, i32, vp, i64, C.c_float, vp, vp, vp, vp, i32, vp, vp, vp, C.c_size_t, vp]
        L.moe_token_logprobs_backward.argtypes = [i32, i32, i32, vp, i64, C.c_float] + [vp] * 7 + [i64, vp]
        _lib = L
    return _lib


def _matrix(x, what: str, shape, dtype, device: int):
    """The address and row stride of a matrix whose rows are contiguous."""
    if x.dim() != 2 or (shape is not None and x.shape != shape) or x.dtype is not dtype:
        raise ValueError(f"{what} is a {x.dtype} tensor of shape {tuple(x.shape)}, the call needs a {dtype} matrix" + (f" of shape {tuple(shape)}" if shape else ""))
    if x.stride(1) != 1 and x.shape[1] > 1:
        raise ValueError(f"{what}: the elements of a row must be contiguous")
    if x.get_device() != device:
        A._wrong_device(what, x, device)
    return x.data_ptr(), x.stride(0)


def moe_token_logprobs_workspace_bytes(T: int, V: int, K: int = 0) -> int:
    n = lib().moe_token_logprobs_workspace_bytes(A._int32(T, "T"), A._int32(V, "V"), A._int32(K, "K"))
    if n == 0:
        raise B.MoEError(1, "moe_token_logprobs_workspace_bytes", lib().moe_last_error().decode())
    return n


def moe_token_logprobs(logits, ids, ws, logp=None, lse=None, entropy=None, top_ids=None, top_logp=None, scale: float = 1.0, stream=None):
    """Outputs for every row of logits [T, V]: logp of ids (int32 [T]), lse, entropy (float32 [T]), top_ids (int32) and top_logp
    (float32) [T, K]."""
    dtype, device = A._dtype(logits), A._device(logits, "logits")
    at, stride = _matrix(logits, "logits", None, logits.dtype, device)
    T, V = logits.shape
    K = 0 if top_ids is None else top_ids.shape[-1]
    if not ws.is_contiguous() or ws.get_device() != device:
        raise ValueError("the workspace must be contiguous and on the logits' device")
    f = lambda t, what: A._vector(t, what, torch.float32, (T,), device)  # noqa: E731
    st = lib().moe_token_logprobs(dtype, A._int32(T, "T"), A._int32(V, "V"), at, stride, scale, A._vector(ids, "ids", torch.int32, (T,), device),
                                  f(logp, "logp"), f(lse, "lse"), f(entropy, "entropy"), A._int32(K, "K"), A._vector(top_ids, "top_ids", torch.int32, (T, K), device),
                                  A._vector(top_logp, "top_logp", torch.float32, (T, K), device), ws.data_ptr(), ws.nbytes, A._stream(stream, device))
    if st:
        B._check(st, "moe_token_logprobs")


def moe_token_logprobs_backward(logits, ids, lse, d_logits, d_logp=None, entropy=None, d_entropy=None, d_lse=None, scale: float = 1.0, stream=None):
    """d_logits [T, V] from the gradients of logp, entropy and lse (float32 [T], None: 0); it may be logits itself."""
    dtype, device = A._dtype(logits), A._device(logits, "logits")
    at, stride = _matrix(logits, "logits", None, logits.dtype, device)
    T, V = logits.shape
    d_at, d_stride = _matrix(d_logits, "d_logits", logits.shape, logits.dtype, device)
    f = lambda t, what: A._vector(t, what, torch.float32, (T,), device)  # noqa: E731
    st = lib().moe_token_logprobs_backward(dtype, A._int32(T, "T"), A._int32(V, "V"), at, stride, scale, A._vector(ids, "ids", torch.int32, (T,), device), f(lse, "lse"),
                                           f(d_logp, "d_logp"), f(entropy, "entropy"), f(d_entropy, "d_entropy"), f(d_lse, "d_lse"), d_at, d_stride,
                                           A._stream(stream, device))
    if st:
        B._check(st, "moe_token_logprobs_backward")
