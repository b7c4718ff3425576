"""The next token of each row from a model's logits: the call of include/ivftq_sample.h on torch tensors.  `stream` as in `kv`."""
from __future__ import annotations

import ctypes as C
import numbers
import struct

import torch

from . import kv
from .binding import _check, load_library

_TYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}


class _Logits(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("rows", C.c_int64), ("vocabulary", C.c_int32), ("type", C.c_int32)]


class _Sampling(C.Structure):
    _fields_ = [("temperature", C.c_void_p), ("top_k", C.c_void_p), ("top_p", C.c_void_p), ("min_p", C.c_void_p), ("temperature_all", C.c_float),
                ("top_k_all", C.c_int32), ("top_p_all", C.c_float), ("min_p_all", C.c_float)]


_P = C.c_void_p
_SIGNATURES = {
    "ivftq_sample_tokens": (C.c_int, [_P, _P, _P, _P, _P, _P, C.c_int64, _P]),
    "ivftq_sample_workspace": (C.c_int64, [_P, _P]),
}

_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)          # AttributeError if the export is missing
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def declared_sample_symbols():
    return list(_SIGNATURES)


_pack_logits, _pack_sampling = kv._packer(_Logits), struct.Struct("@PPPPfiff").pack


def _setting(v, name, like, rows, dtype):
    """(pointer, value): an array with a value for each row, or one value for all."""
    if not isinstance(v, torch.Tensor):
        return 0, v
    kv._on_device(v, name, like)
    if v.dtype != dtype or v.shape != (rows,) or not v.is_contiguous():
        raise ValueError(f"{name} must be a number or a contiguous {dtype} tensor of ({rows},), got {tuple(v.shape)} in {v.dtype}")
    return v.data_ptr(), 0


def _settings(*values):
    """The library's structure; values: pointers, then the numbers for all rows in its order."""
    try:
        return _pack_sampling(*values)
    except (struct.error, TypeError, OverflowError):
        for name, v, kind in zip(("temperature", "top_k", "top_p", "min_p"), values[4:], (numbers.Real, numbers.Integral, numbers.Real, numbers.Real)):
            if not isinstance(v, kind):
                raise TypeError(f"{name} must be a {'whole ' if kind is numbers.Integral else ''}number, or a tensor with a value for each row, got {v!r}") from None
        raise ValueError("temperature = {!r}, top_k = {!r}, top_p = {!r}, min_p = {!r}: one does not fit 32 bits".format(*values[4:])) from None


def sample_tokens(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, out=None, logprobs=None, stream=None):
    """Tokens, int32 [rows], of logits [rows, vocabulary] in float32, float16 or bfloat16; u: float32 [rows] from [0, 1).

    Weights are w = e^((x - max x) / temperature).  Ranked by x (ties: the lowest index) the first top_k are kept (0: all), of these the ranks
    before which there is less than top_p of their mass, of these the ones with w >= min_p; the token is the lowest index up to which the kept
    weights pass u times their sum.  temperature 0: the largest logit.  Settings are numbers, or tensors with a value for each row
    (float32; top_k int32).  logprobs (float32 [rows], optional) receives the logarithm of the token's probability among the kept
    ones.  A row without a finite or infinite logit above -inf gives -1."""
    kv._on_device(logits, "logits")
    if logits.requires_grad:
        kv._no_gradient(logits, "logits")
    kind = _TYPES.get(logits.dtype)
    if kind is None:
        raise TypeError(f"logits must be float32, float16 or bfloat16, got {logits.dtype}")
    if logits.dim() != 2 or (logits.stride(1) != 1 and logits.shape[1] > 1 and logits.numel()):
        raise ValueError(f"logits must be rows x vocabulary with neighbouring tokens, got {tuple(logits.shape)} with strides {logits.stride()}")
    (rows, vocabulary), where = logits.shape, kv._stream(stream, logits)
    data = _pack_logits(logits.data_ptr(), logits.stride(0) if rows > 1 else vocabulary, rows, vocabulary, kind)
    t, t_all = _setting(temperature, "temperature", logits, rows, torch.float32)
    k, k_all = _setting(top_k, "top_k", logits, rows, torch.int32)
    p, p_all = _setting(top_p, "top_p", logits, rows, torch.float32)
    m, m_all = _setting(min_p, "min_p", logits, rows, torch.float32)
    how, draws = _settings(t, k, p, m, t_all, k_all, p_all, m_all), kv._floats(u, "u", logits, (rows,))
    if out is None:
        out = kv._blank(rows, torch.int32, logits, stream)
    result, logs = kv._ints(out, "out", logits, rows), None if logprobs is None else kv._floats(logprobs, "logprobs", logits, (rows,))
    lib = _library()
    need = lib.ivftq_sample_workspace(data, how)
    if need < 0:
        _check(1)
    work = kv._scratch(need, torch.uint8, logits, stream) if need else None
    kv._run(lib.ivftq_sample_tokens, logits, data, draws, how, result, logs, None if work is None else work.data_ptr(), need, where)
    return out
