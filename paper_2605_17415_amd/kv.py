"""Paged key-value cache: the calls of include/ivftq_kv.h on torch tensors, and `KVCache`, which keeps a model's cache.

Like `binding`, this module marshals arguments; every step runs in the library's HIP kernels.  A pool holds one layer:
    16 bits   float16 / bfloat16 [pages, heads, 2, page, d]   keys [page][d], then values in groups of eight tokens:
              the second block is really [page / 8][d][8]
    codes     uint8 [pages, heads, page * (d + 4)]            see ivftq_kv.h
and tensors of several layers have one more dimension in front.
"""
from __future__ import annotations

import ctypes as C
import math

import numpy as np

from .binding import _check, _np_ptr, ivftq_build_codebook, ivftq_haar_rotation, load_library

F16, BF16, CODE4 = range(3)
HEAD_SIZES = (64, 96, 128, 192, 256)


class _Cache(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("table", C.c_void_p), ("lengths", C.c_void_p), ("rotation", C.c_void_p), ("pages", C.c_int64),
                ("table_stride", C.c_int64), ("batch", C.c_int32), ("columns", C.c_int32), ("format", C.c_int32), ("page", C.c_int32),
                ("heads", C.c_int32), ("d", C.c_int32), ("levels", C.c_float * 16)]


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64), ("rows", C.c_int64), ("heads", C.c_int32),
                ("type", C.c_int32)]


class _Pages(C.Structure):
    _fields_ = [("table", C.c_void_p), ("lengths", C.c_void_p), ("refs", C.c_void_p), ("table_stride", C.c_int64), ("pages", C.c_int64),
                ("rows", C.c_int32), ("columns", C.c_int32), ("page", C.c_int32)]


class _Pools(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("layer_stride", C.c_int64), ("page_bytes", C.c_int64), ("pages", C.c_int64), ("layers", C.c_int32)]


_P = C.c_void_p
_SIGNATURES = {
    "ivftq_kv_page_bytes": (C.c_int64, [C.c_int, C.c_int, C.c_int, C.c_int]),
    "ivftq_kv_append": (C.c_int, [C.POINTER(_Cache), C.POINTER(_Rows), C.POINTER(_Rows), _P, _P]),
    "ivftq_kv_read": (C.c_int, [C.POINTER(_Cache), C.POINTER(_Rows), C.POINTER(_Rows), _P, _P]),
    "ivftq_kv_attend": (C.c_int, [C.POINTER(_Cache), C.POINTER(_Rows), C.POINTER(_Rows), _P, _P, C.c_int32, C.c_int32, C.c_int32, C.c_float,
                                  _P, C.c_int64, _P]),
    "ivftq_kv_attend_workspace": (C.c_int64, [C.POINTER(_Cache), C.c_int64, C.c_int32, C.c_int32]),
    "ivftq_kv_reserve": (C.c_int, [C.POINTER(_Pages), _P, _P, _P, _P]),
    "ivftq_kv_fork": (C.c_int, [C.POINTER(_Pages), C.POINTER(_Pools), _P, _P, C.c_int32, _P, _P, _P]),
    "ivftq_kv_free": (C.c_int, [C.POINTER(_Pages), _P, C.c_int32, _P]),
    "ivftq_kv_trim": (C.c_int, [C.POINTER(_Pages), C.c_int32, C.c_int32, _P]),
    "ivftq_kv_compact": (C.c_int, [C.POINTER(_Pages), C.POINTER(_Pools), _P, _P, _P]),
    "ivftq_kv_copy": (C.c_int, [C.POINTER(_Pools), _P, _P, C.c_int32, _P]),
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


def declared_kv_symbols():
    return list(_SIGNATURES)


def kv_page_bytes(format: int, page: int, heads: int, d: int) -> int:
    return _library().ivftq_kv_page_bytes(format, page, heads, d)


# ---- arguments -----------------------------------------------------------------------------------


def _on_device(t, name, like=None):
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a torch tensor in device memory")
    if like is not None and t.device != like.device:
        raise ValueError(f"{name} is on {t.device}, not on {like.device}")


def _ints(t, name, like, shape=None):
    """Pointer of a contiguous int32 tensor on `like`'s device (None -> NULL)."""
    import torch
    if t is None:
        return None
    _on_device(t, name, like)
    if t.dtype != torch.int32 or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous int32 tensor")
    if shape is not None and tuple(t.shape) != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {shape}")
    return t.data_ptr()


def _table(table, like):
    import torch
    _on_device(table, "table", like)
    if table.dtype != torch.int32 or table.dim() != 2 or (table.numel() and table.stride(1) != 1):
        raise TypeError("table must be an int32 matrix with neighbouring columns")
    return table.data_ptr(), table.stride(0) if table.shape[0] > 1 else table.shape[1]


def _type_of(t, name):
    import torch
    if t.dtype == torch.float16:
        return F16
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"{name} must be float16 or bfloat16, got {t.dtype}")


def _rows(t, name, like, d):
    _on_device(t, name, like)
    if t.dim() != 3 or t.shape[2] != d:
        raise ValueError(f"{name} must be rows x heads x {d}, got {tuple(t.shape)}")
    if t.stride(2) != 1 and t.numel():
        raise ValueError(f"{name}: the coordinates of a row must be neighbours")
    return _Rows(t.data_ptr(), t.stride(0), t.stride(1), t.shape[0], t.shape[1], _type_of(t, name))


def _cache(pool, table, lengths, d, rotation, levels):
    import torch
    _on_device(pool, "pool")
    if not pool.is_contiguous():
        raise ValueError("pool must be contiguous")
    if pool.dtype == torch.uint8:
        if pool.dim() != 3 or pool.shape[2] % (d + 4):
            raise ValueError(f"a pool of codes is pages x heads x page * (d + 4) bytes, got {tuple(pool.shape)} for d = {d}")
        form, page = CODE4, pool.shape[2] // (d + 4)
        _on_device(rotation, "rotation", pool)
        if rotation.dtype != torch.float32 or tuple(rotation.shape) != (d, d) or not rotation.is_contiguous():
            raise ValueError(f"rotation must be a contiguous float32 matrix of {d} x {d}")
        levels = np.ascontiguousarray(levels, np.float32)
        if levels.shape != (16,):
            raise ValueError("levels must be 16 numbers")
        turn, values = rotation.data_ptr(), (C.c_float * 16).from_buffer_copy(levels)
    else:
        if pool.dim() != 5 or pool.shape[2] != 2 or pool.shape[4] != d:
            raise ValueError(f"a 16-bit pool is pages x heads x 2 x page x {d}, got {tuple(pool.shape)}")
        form, page, turn, values = _type_of(pool, "pool"), pool.shape[3], None, (C.c_float * 16)()
    where, stride = _table(table, pool)
    return _Cache(pool.data_ptr(), where, _ints(lengths, "lengths", pool, (table.shape[0],)), turn, pool.shape[0], stride, table.shape[0], table.shape[1], form, page, pool.shape[1], d, values)


def _starts(starts, table, like):
    return _ints(starts, "starts", like, (table.shape[0] + 1,))


def _stream(stream, like):
    import torch
    return (stream if stream is not None else torch.cuda.current_stream(like.device)).cuda_stream


class _Scratch:
    """Device memory for the length of a call: from the caching allocator, marked as used by the call's stream."""

    def __new__(cls, nbytes, like, stream):
        import torch
        t = torch.empty(nbytes, dtype=torch.uint8, device=like.device)
        if stream is not None:
            t.record_stream(stream)
        return t


# ---- rows and attention --------------------------------------------------------------------------


def kv_append(pool, k, v, table, lengths, starts=None, rotation=None, levels=None, stream=None):
    """Write the new rows k, v [rows, heads, d] of every sequence to its pages: sequence b's rows are starts[b] ..
    starts[b + 1] - 1 and its last tokens (starts None: one row per sequence).  lengths count the new tokens already."""
    lib = _library()
    d = k.shape[-1]
    _check(lib.ivftq_kv_append(C.byref(_cache(pool, table, lengths, d, rotation, levels)), C.byref(_rows(k, "k", pool, d)),
                               C.byref(_rows(v, "v", pool, d)), _starts(starts, table, pool), _stream(stream, pool)))


def kv_read(pool, table, lengths, k_out, v_out, starts=None, rotation=None, levels=None, stream=None):
    """The opposite of kv_append: the rows that the cache holds for these tokens."""
    lib = _library()
    d = k_out.shape[-1]
    _check(lib.ivftq_kv_read(C.byref(_cache(pool, table, lengths, d, rotation, levels)), C.byref(_rows(k_out, "k_out", pool, d)),
                             C.byref(_rows(v_out, "v_out", pool, d)), _starts(starts, table, pool), _stream(stream, pool)))


def kv_attend(q, pool, table, lengths, starts=None, max_new=1, window=0, sinks=0, scale=None, rotation=None, levels=None, out=None,
              lse=None, stream=None):
    """Attention of the new rows q [rows, query heads, d] over the cache; returns out (like q).  The last rows of a sequence are
    its last tokens; a token sees itself and those before it, with a window the last `window` of them and the first `sinks`.
    max_new: no sequence has more new rows.  lse (float32 [rows, query heads], optional) receives the logarithm of the sums."""
    import torch
    lib = _library()
    d = q.shape[-1]
    cache, rows = _cache(pool, table, lengths, d, rotation, levels), _rows(q, "q", pool, d)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if stream is not None:
            out.record_stream(stream)
    elif tuple(out.shape) != tuple(q.shape):
        raise ValueError(f"out has shape {tuple(out.shape)}, not {tuple(q.shape)}")
    result = _rows(out, "out", pool, d)
    if lse is not None:
        _on_device(lse, "lse", pool)
        if lse.dtype != torch.float32 or tuple(lse.shape) != tuple(q.shape[:2]) or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous float32 matrix of rows x query heads")
    first = _starts(starts, table, pool)
    need = lib.ivftq_kv_attend_workspace(C.byref(cache), rows.rows, rows.heads, max_new)
    if need < 0:
        _check(1)
    work = _Scratch(need, q, stream) if need else None
    _check(lib.ivftq_kv_attend(C.byref(cache), C.byref(rows), C.byref(result), None if lse is None else lse.data_ptr(), first, max_new, window,
                               sinks, 1 / math.sqrt(d) if scale is None else scale, None if work is None else work.data_ptr(), need,
                               _stream(stream, pool)))
    return out


# ---- pages ---------------------------------------------------------------------------------------


def _pages(table, lengths, refs, page):
    _on_device(refs, "refs")
    where, stride = _table(table, refs)
    return _Pages(where, _ints(lengths, "lengths", refs, (table.shape[0],)), _ints(refs, "refs", refs, (refs.numel(),)), stride, refs.numel(), table.shape[0], table.shape[1], page)


def _pools(pools, like):
    """[layers, pages, ...]: contiguous records, layers any distance apart."""
    _on_device(pools, "pools", like)
    if pools.dim() < 3 or (pools.numel() and not pools[0].is_contiguous()):
        raise ValueError("pools must be layers x pages x record with contiguous layers")
    size = pools.element_size()
    return _Pools(pools.data_ptr(), pools.stride(0) * size, pools[0, 0].numel() * size, pools.shape[1], pools.shape[0])


def _like(t, stream, count=None):
    import torch
    r = torch.empty(t.numel() if count is None else count, dtype=torch.int32, device=t.device)
    if stream is not None:
        r.record_stream(stream)
    return r


def kv_reserve(table, lengths, refs, counts, page, stream=None):
    """Pages for counts[r] more tokens in each row, lengths raised; returns what was granted (counts[r] or 0)."""
    state = _pages(table, lengths, refs, page)
    granted, scratch = _like(lengths, stream), _like(refs, stream)
    _check(_library().ivftq_kv_reserve(C.byref(state), _ints(counts, "counts", refs, tuple(lengths.shape)), granted.data_ptr(), scratch.data_ptr(),
                                       _stream(stream, refs)))
    return granted


def kv_fork(pools, table, lengths, refs, parents, children, page, stream=None):
    """Rows `children` become copies of rows `parents`: full pages shared, a last page that is not full copied in every layer
    of pools [layers, pages, ...].  Returns 1 for each entry that was done."""
    state, where = _pages(table, lengths, refs, page), _pools(pools, refs)
    n = parents.numel()
    done, scratch = _like(parents, stream), _like(refs, stream, refs.numel() + 2 * n + 2 * table.shape[0])
    _check(_library().ivftq_kv_fork(C.byref(state), C.byref(where), _ints(parents, "parents", refs), _ints(children, "children", refs, (n,)), n,
                                    done.data_ptr(), scratch.data_ptr(), _stream(stream, refs)))
    return done


def kv_free(table, lengths, refs, rows, stream=None):
    """Rows give their pages back and become empty."""
    state = _pages(table, lengths, refs, 16)
    _check(_library().ivftq_kv_free(C.byref(state), _ints(rows, "rows", refs), rows.numel(), _stream(stream, refs)))


def kv_trim(table, lengths, refs, page, window, sinks=0, stream=None):
    """Every row gives back the pages that no later token sees with this window and these first tokens."""
    state = _pages(table, lengths, refs, page)
    _check(_library().ivftq_kv_trim(C.byref(state), window, sinks, _stream(stream, refs)))


def kv_compact(pools, table, refs, stream=None):
    """Pages in use move to the lowest numbers; returns how many there are (device, int32 [1])."""
    state, where = _pages(table, None, refs, 16), _pools(pools, refs)
    used, scratch = _like(refs, stream, 1), _like(refs, stream, 3 * refs.numel() + 64)
    _check(_library().ivftq_kv_compact(C.byref(state), C.byref(where), used.data_ptr(), scratch.data_ptr(), _stream(stream, refs)))
    return used


def kv_copy(pools, src, dst, stream=None):
    """Record of page src[i] to page dst[i] in every layer of pools; no page both source and destination."""
    where = _pools(pools, pools)
    _check(_library().ivftq_kv_copy(C.byref(where), _ints(src, "src", pools), _ints(dst, "dst", pools, tuple(src.shape)), src.numel(),
                                    _stream(stream, pools)))
