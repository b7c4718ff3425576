"""Paged key-value cache: the calls of include/ivftq_kv.h on torch tensors, and `KVCache`, which keeps a model's cache.

Like `binding`, this module marshals arguments; every step runs in the library's HIP kernels.  A pool holds one layer:
    16 bits   float16 / bfloat16 [pages, heads, 2, page, d]   keys [page][d], then values in groups of eight tokens:
              the second block is really [page / 8][d][8]
    codes     uint8 [pages, heads, page * (d + 4)]            see ivftq_kv.h
and its digests, the lowest and the highest value of a page's key coordinates, by which pages are chosen for attention over a long cache:
    digests   [pages, heads, 2, d] of the pool's type (codes: float16, of the rotated keys)
and tensors of several layers have one more dimension in front.

`stream`: a call's kernels, its workspace and what it gives back belong to this stream (None: the current one).  As everywhere in
PyTorch the caller has `stream` wait for the work that makes the inputs, and the reader of results wait for `stream`; inputs from
another stream that are dropped while the call is queued are the caller's to record.

The cache serves: there is no backward pass, and rows that ask for a gradient are refused unless gradients are off.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import math
import struct

import numpy as np
import torch

from .binding import _check, ivftq_build_codebook, ivftq_haar_rotation, load_library

F16, BF16, CODE4 = range(3)
HEAD_SIZES = (64, 96, 128, 192, 256)
MOST_PICKS = 4096           # pages that a row and key-value head can be given
_TYPES = {torch.float16: F16, torch.bfloat16: BF16}


class _Cache(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("table", C.c_void_p), ("lengths", C.c_void_p), ("rotation", C.c_void_p), ("pages", C.c_int64),
                ("table_stride", C.c_int64), ("batch", C.c_int32), ("columns", C.c_int32), ("format", C.c_int32), ("page", C.c_int32),
                ("heads", C.c_int32), ("d", C.c_int32), ("levels", C.c_float * 16), ("asked", C.c_void_p), ("granted", C.c_void_p)]


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64), ("rows", C.c_int64), ("heads", C.c_int32),
                ("type", C.c_int32)]


class _Pages(C.Structure):
    _fields_ = [("table", C.c_void_p), ("lengths", C.c_void_p), ("refs", C.c_void_p), ("table_stride", C.c_int64), ("pages", C.c_int64),
                ("rows", C.c_int32), ("columns", C.c_int32), ("page", C.c_int32)]


class _Pools(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("layer_stride", C.c_int64), ("page_bytes", C.c_int64), ("pages", C.c_int64), ("layers", C.c_int32)]


# A call's structures are packed as bytes, a third of the time that ctypes takes to fill one in.
_CODES = {C.c_void_p: "P", C.c_int64: "q", C.c_int32: "i"}


def _packer(cls):
    return struct.Struct("@" + "".join(_CODES.get(t) or f"{C.sizeof(t)}s" for _, t in cls._fields_) + "0q").pack


_pack_cache, _pack_rows, _pack_pages, _pack_pools = (_packer(c) for c in (_Cache, _Rows, _Pages, _Pools))
_NO_LEVELS = bytes(64)

_P = C.c_void_p
_SIGNATURES = {
    "ivftq_kv_page_bytes": (C.c_int64, [C.c_int, C.c_int, C.c_int, C.c_int]),
    "ivftq_kv_append": (C.c_int, [_P, _P, _P, _P, _P]),
    "ivftq_kv_read": (C.c_int, [_P, _P, _P, _P, _P]),
    "ivftq_kv_attend": (C.c_int, [_P, _P, _P, _P, _P, C.c_int32, C.c_int32, C.c_int32, C.c_float,
                                  _P, C.c_int64, _P]),
    "ivftq_kv_attend_workspace": (C.c_int64, [_P, C.c_int64, C.c_int32, C.c_int32]),
    "ivftq_kv_digest": (C.c_int, [_P, _P, _P, _P]),
    "ivftq_kv_score": (C.c_int, [_P, _P, _P, _P, _P, C.c_int32, _P, C.c_int64, _P]),
    "ivftq_kv_score_workspace": (C.c_int64, [_P, C.c_int64, C.c_int32, C.c_int32]),
    "ivftq_kv_select": (C.c_int, [_P, _P, _P, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _P, _P]),
    "ivftq_kv_attend_pages": (C.c_int, [_P, _P, _P, _P, _P, C.c_int32, _P, C.c_int32, C.c_float, _P, C.c_int64, _P]),
    "ivftq_kv_attend_pages_workspace": (C.c_int64, [_P, C.c_int64, C.c_int32, C.c_int32, C.c_int32]),
    "ivftq_kv_reserve": (C.c_int, [_P, _P, _P, _P, _P]),
    "ivftq_kv_fork": (C.c_int, [_P, _P, _P, _P, C.c_int32, _P, _P, _P]),
    "ivftq_kv_fork_pools": (C.c_int, [_P, _P, C.c_int32, _P, _P, C.c_int32, _P, _P, _P]),
    "ivftq_kv_compact_pools": (C.c_int, [_P, _P, C.c_int32, _P, _P, _P]),
    "ivftq_kv_free": (C.c_int, [_P, _P, C.c_int32, _P]),
    "ivftq_kv_trim": (C.c_int, [_P, C.c_int32, C.c_int32, _P]),
    "ivftq_kv_compact": (C.c_int, [_P, _P, _P, _P, _P]),
    "ivftq_kv_copy": (C.c_int, [_P, _P, _P, C.c_int32, _P]),
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
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a torch tensor in device memory")
    if like is not None and t.get_device() != like.get_device():
        raise ValueError(f"{name} is on {t.device}, not on {like.device}")


def _ints(t, name, like, count=None):
    """Pointer of a contiguous vector of int32 on `like`'s device (None -> NULL)."""
    if t is None:
        return None
    _on_device(t, name, like)
    if t.dtype != torch.int32 or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous int32 tensor")
    if t.dim() != 1 or (count is not None and t.shape[0] != count):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not ({'n' if count is None else count},)")
    return t.data_ptr()


def _table(table, like):
    _on_device(table, "table", like)
    if table.dtype != torch.int32 or table.dim() != 2 or (table.stride(1) != 1 and table.numel()):
        raise TypeError("table must be an int32 matrix with neighbouring columns")
    rows, columns = table.shape
    return table.data_ptr(), table.stride(0) if rows > 1 else columns, rows, columns


def _type_of(t, name):
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise TypeError(f"{name} must be float16 or bfloat16, got {t.dtype}")
    return kind


def _no_gradient(t, name):
    if torch.is_grad_enabled():
        raise ValueError(f"{name} asks for a gradient, and the cache's calls have none: call them under torch.no_grad()")


def _rows(t, name, like, d):
    _on_device(t, name, like)
    if t.requires_grad:
        _no_gradient(t, name)
    if t.dim() != 3 or t.shape[2] != d:
        raise ValueError(f"{name} must be rows x heads x {d}, got {tuple(t.shape)}")
    row, head, one = t.stride()
    rows, heads, _ = t.shape
    if one != 1 and t.numel():
        raise ValueError(f"{name}: the coordinates of a row must be neighbours")
    return _pack_rows(t.data_ptr(), row, head, rows, heads, _type_of(t, name))


def _cache(pool, table, lengths, d, rotation, levels, asked=None, granted=None):
    _on_device(pool, "pool")
    if pool.requires_grad:
        _no_gradient(pool, "pool")
    if not pool.is_contiguous():
        raise ValueError("pool must be contiguous")
    shape, turn, values = pool.shape, 0, _NO_LEVELS
    if pool.dtype == torch.uint8:
        if len(shape) != 3 or shape[2] % (d + 4):
            raise ValueError(f"a pool of codes is pages x heads x page * (d + 4) bytes, got {tuple(shape)} for d = {d}")
        form, page = CODE4, shape[2] // (d + 4)
        _on_device(rotation, "rotation", pool)
        if rotation.dtype != torch.float32 or tuple(rotation.shape) != (d, d) or not rotation.is_contiguous():
            raise ValueError(f"rotation must be a contiguous float32 matrix of {d} x {d}")
        turn, values = rotation.data_ptr(), np.asarray(levels, np.float32).tobytes()
        if len(values) != 64:
            raise ValueError("levels must be 16 numbers")
    else:
        if len(shape) != 5 or shape[2] != 2 or shape[4] != d:
            raise ValueError(f"a 16-bit pool is pages x heads x 2 x page x {d}, got {tuple(shape)}")
        form, page = _type_of(pool, "pool"), shape[3]
    where, stride, batch, columns = _table(table, pool)
    return _pack_cache(pool.data_ptr(), where, _ints(lengths, "lengths", pool, batch), turn, shape[0], stride, batch, columns, form, page, shape[1], d, values,
                       0 if asked is None else _ints(asked, "asked", pool, batch), 0 if granted is None else _ints(granted, "granted", pool, batch))


def _starts(starts, table, like):
    return None if starts is None else _ints(starts, "starts", like, table.shape[0] + 1)


def _stream(stream, like):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(like.device.index)
    if stream.device != like.device:
        raise ValueError(f"the stream is of {stream.device}, the tensors are on {like.device}")
    return stream.cuda_stream


def _run(call, like, *args):
    """The library launches on the current device, which has to be that of the tensors."""
    if like.device.index == torch._C._cuda_getDevice():
        _check(call(*args))
    else:
        with torch.cuda.device(like.device):
            _check(call(*args))


def _scratch(count, dtype, like, stream):
    """Device memory from the caching allocator's share of the stream that uses it: the current stream may still use what it has freed."""
    if stream is None:
        return like.new_empty(count, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(count, dtype=dtype)


def _result(t, stream):
    """A tensor that is given back, made for `stream`: the caller's current stream reads it, and its memory waits for that."""
    if stream is not None:
        t.record_stream(torch.cuda.current_stream(t.device))
    return t


# ---- rows and attention --------------------------------------------------------------------------


def kv_append(pool, k, v, table, lengths, starts=None, rotation=None, levels=None, stream=None, asked=None, granted=None):
    """Write the new rows k, v [rows, heads, d] of every sequence to its pages: sequence b's rows are starts[b] ..
    starts[b + 1] - 1 and its last tokens (starts None: one row per sequence).  lengths count the new tokens already, unless
    kv_reserve refused them: with its counts as `asked` and its result as `granted`, such sequences' rows are not written (without
    the two they fall on the tokens before them)."""
    d = k.shape[-1]
    _run(_library().ivftq_kv_append, pool, _cache(pool, table, lengths, d, rotation, levels, asked, granted), _rows(k, "k", pool, d), _rows(v, "v", pool, d),
         _starts(starts, table, pool), _stream(stream, pool))


def kv_read(pool, table, lengths, k_out, v_out, starts=None, rotation=None, levels=None, stream=None):
    """The opposite of kv_append: the rows that the cache holds for these tokens."""
    d = k_out.shape[-1]
    _run(_library().ivftq_kv_read, pool, _cache(pool, table, lengths, d, rotation, levels), _rows(k_out, "k_out", pool, d), _rows(v_out, "v_out", pool, d),
         _starts(starts, table, pool), _stream(stream, pool))


def kv_attend(q, pool, table, lengths, starts=None, max_new=None, window=0, sinks=0, scale=None, rotation=None, levels=None, out=None,
              lse=None, stream=None):
    """Attention of the new rows q [rows, query heads, d] over the cache; returns out (like q).  The last rows of a sequence are
    its last tokens; a token sees itself and those before it, with a window the last `window` of them and the first `sinks`.
    max_new: no sequence has more new rows (None: whatever number; a call that is told prepares for fewer).  Rows past it and rows of no
    sequence keep what `out` holds, which is nothing in particular where it is not given.  lse (float32 [rows, query heads], optional) receives the logarithm of the sums."""
    lib = _library()
    d = q.shape[-1]
    cache, rows, where = _cache(pool, table, lengths, d, rotation, levels), _rows(q, "q", pool, d), _stream(stream, pool)
    if out is None:
        if stream is None:
            out = torch.empty_like(q)
        else:
            with torch.cuda.stream(stream):
                out = torch.empty_like(q)
            _result(out, stream)
    elif out.shape != q.shape:
        raise ValueError(f"out has shape {tuple(out.shape)}, not {tuple(q.shape)}")
    result = _rows(out, "out", pool, d)
    if lse is not None:
        _on_device(lse, "lse", pool)
        if lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous float32 matrix of rows x query heads")
    first = _starts(starts, table, pool)
    if starts is None and (max_new is None or max_new > 1):
        max_new = 1
    elif max_new is None:
        max_new = max(q.shape[0], 1)
    need = lib.ivftq_kv_attend_workspace(cache, q.shape[0], q.shape[1], max_new)
    if need < 0:
        _check(1)
    work = _scratch(need, torch.uint8, q, stream) if need else None
    _run(lib.ivftq_kv_attend, pool, cache, rows, result, None if lse is None else lse.data_ptr(), first, max_new, window, sinks,
         1 / math.sqrt(d) if scale is None else scale, None if work is None else work.data_ptr(), need, where)
    return out


# ---- attention over chosen pages ------------------------------------------------------------------


def _digests(digests, pool, d):
    _on_device(digests, "digests", pool)
    if digests.requires_grad:
        _no_gradient(digests, "digests")
    kind = torch.float16 if pool.dtype == torch.uint8 else pool.dtype
    if digests.dtype != kind or digests.shape != (*pool.shape[:2], 2, d) or not digests.is_contiguous():
        raise ValueError(f"digests must be a contiguous tensor of pages x heads x 2 x {d} in {kind}, got {tuple(digests.shape)} in {digests.dtype}")
    return digests.data_ptr()


def _floats(t, name, like, shape):
    _on_device(t, name, like)
    if t.requires_grad:
        _no_gradient(t, name)
    if t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 tensor of {tuple(shape)}, got {tuple(t.shape)} in {t.dtype}")
    return t.data_ptr()


def _most_new(max_new, starts, rows):
    if starts is None and (max_new is None or max_new > 1):
        return 1
    return max(rows, 1) if max_new is None else max_new


def _blank(shape, dtype, like, stream):
    """A tensor that is given back."""
    return like.new_empty(shape, dtype=dtype) if stream is None else _result(_scratch(shape, dtype, like, stream), stream)


def kv_digest(pool, digests, table, lengths, starts=None, rotation=None, levels=None, stream=None, asked=None, granted=None):
    """Digests of the pages that hold the new rows, after kv_append has written them (and with its starts, asked and granted): a page that
    begins with a new row gets the digest of its new rows, one that goes on has them added.  With all of a sequence's tokens between
    its starts its digests are made afresh."""
    _on_device(digests, "digests")
    d = digests.shape[-1]
    where = _digests(digests, pool, d)
    _run(_library().ivftq_kv_digest, pool, _cache(pool, table, lengths, d, rotation, levels, asked, granted), where, _starts(starts, table, pool), _stream(stream, pool))


def kv_score(q, digests, pool, table, lengths, starts=None, max_new=None, rotation=None, levels=None, out=None, stream=None):
    """Scores of every page for the new rows q [rows, query heads, d]: float32 [rows, heads, columns], for each key-value head the most that
    the products of its query heads with a key of the page can add up to (-inf: the row sees nothing of it; inf: one of the page's keys is
    infinite).  What is no number in every key counts for nothing, and so does a query's coordinate that is no finite number.  max_new and rows
    past it as in kv_attend."""
    d = q.shape[-1]
    cache, rows, where = _cache(pool, table, lengths, d, rotation, levels), _rows(q, "q", pool, d), _stream(stream, pool)
    box, shape = _digests(digests, pool, d), (q.shape[0], pool.shape[1], table.shape[1])
    if out is None:
        out = _blank(shape, torch.float32, q, stream)
    result, first, max_new = _floats(out, "out", pool, shape), _starts(starts, table, pool), _most_new(max_new, starts, q.shape[0])
    lib = _library()
    need = 0 if max_new == 1 and pool.dtype != torch.uint8 else lib.ivftq_kv_score_workspace(cache, q.shape[0], q.shape[1], max_new)
    if need < 0:
        _check(1)
    work = _scratch(need, torch.uint8, q, stream) if need else None
    _run(lib.ivftq_kv_score, pool, cache, rows, box, result, first, max_new, None if work is None else work.data_ptr(), need, where)
    return out


def kv_select(scores, lengths, page, count, starts=None, first=1, last=1, out=None, stream=None):
    """The pages of each row and key-value head: int32 [rows, heads, count], of the columns that the row's position reaches the first `first`
    and the last `last` ones and those of the highest scores (ties: the lowest column; -inf and what is no number: none), ascending, -1
    behind them."""
    _on_device(scores, "scores")
    if scores.dim() != 3:
        raise ValueError(f"scores must be rows x heads x columns, got {tuple(scores.shape)}")
    rows, heads, columns = scores.shape
    data, where = _floats(scores, "scores", scores, scores.shape), _stream(stream, scores)
    _on_device(lengths, "lengths", scores)
    lens, batch = _ints(lengths, "lengths", scores), lengths.shape[0]
    if not 1 <= count <= MOST_PICKS:
        raise ValueError(f"count = {count}: 1 to {MOST_PICKS}")
    if out is None:
        out = _blank((rows, heads, count), torch.int32, scores, stream)
    _run(_library().ivftq_kv_select, scores, data, lens, None if starts is None else _ints(starts, "starts", scores, batch + 1), rows, batch, heads, columns, page, count,
         first, last, _columns(out, "out", scores, (rows, heads, count)), where)
    return out


def _columns(t, name, like, shape):
    _on_device(t, name, like)
    if t.dtype != torch.int32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor of {tuple(shape)}, got {tuple(t.shape)} in {t.dtype}")
    return t.data_ptr()


def kv_attend_pages(q, pool, table, lengths, chosen, starts=None, max_new=None, scale=None, rotation=None, levels=None, out=None, lse=None, stream=None):
    """kv_attend where a row and key-value head sees, of the tokens up to its own, those of the columns `chosen` [rows, heads, count] (as
    kv_select gives them: ascending; an entry that is not above those before it, or names no page, is passed over)."""
    lib = _library()
    d = q.shape[-1]
    cache, rows, where = _cache(pool, table, lengths, d, rotation, levels), _rows(q, "q", pool, d), _stream(stream, pool)
    _on_device(chosen, "chosen", pool)
    if chosen.dim() != 3:
        raise ValueError(f"chosen must be rows x heads x count, got {tuple(chosen.shape)}")
    count = chosen.shape[2]
    pages = _columns(chosen, "chosen", pool, (q.shape[0], pool.shape[1], count))
    if out is None:
        out = _blank(q.shape, q.dtype, q, stream)
    elif out.shape != q.shape:
        raise ValueError(f"out has shape {tuple(out.shape)}, not {tuple(q.shape)}")
    result, sums = _rows(out, "out", pool, d), None if lse is None else _floats(lse, "lse", pool, q.shape[:2])
    first, max_new = _starts(starts, table, pool), _most_new(max_new, starts, q.shape[0])
    need = lib.ivftq_kv_attend_pages_workspace(cache, q.shape[0], q.shape[1], max_new, count)
    if need < 0:
        _check(1)
    work = _scratch(need, torch.uint8, q, stream) if need else None
    _run(lib.ivftq_kv_attend_pages, pool, cache, rows, result, sums, first, max_new, pages, count, 1 / math.sqrt(d) if scale is None else scale,
         None if work is None else work.data_ptr(), need, where)
    return out


# ---- pages ---------------------------------------------------------------------------------------


def _pages(table, lengths, refs, page):
    where, stride, rows, columns = _table(table, refs)
    return _pack_pages(where, 0 if lengths is None else _ints(lengths, "lengths", refs, rows), _ints(refs, "refs", refs), stride, refs.numel(), rows, columns, page)


def _pools(pools, like):
    """[layers, pages, ...]: contiguous records, layers any distance apart."""
    _on_device(pools, "pools", like)
    if pools.dim() < 3 or not pools.numel() or not (pools.is_contiguous() or pools[0].is_contiguous()):
        raise ValueError("pools must be layers x pages x record with contiguous layers")
    size, (layers, pages) = pools.element_size(), pools.shape[:2]
    return _pack_pools(pools.data_ptr(), pools.stride(0) * size, pools.numel() // (layers * pages) * size, pages, layers)


def _groups(pools, like):
    """(structures of all tensors, their number)"""
    if isinstance(pools, torch.Tensor):
        return _pools(pools, like), 1
    return b"".join(_pools(p, like) for p in pools), len(pools)


def kv_reserve(table, lengths, refs, counts, page, stream=None):
    """Pages for counts[r] more tokens in each row, lengths raised; returns what was granted (counts[r], or 0 where there is no
    room: the row stays as it is, and new rows must not be appended to it)."""
    state, rows, where = _pages(table, lengths, refs, page), table.shape[0], _stream(stream, refs)
    granted, scratch = _result(_scratch(rows, torch.int32, refs, stream), stream), _scratch(refs.numel(), torch.int32, refs, stream)
    _run(_library().ivftq_kv_reserve, refs, state, _ints(counts, "counts", refs, rows), granted.data_ptr(), scratch.data_ptr(), where)
    return granted


def kv_fork(pools, table, lengths, refs, parents, children, page, stream=None):
    """Rows `children` become copies of rows `parents`: full pages shared, a last page that is not full copied in every layer
    of pools [layers, pages, ...] (several such tensors: a list of them).  Returns 1 for each entry that was done."""
    state, records, n, where = _pages(table, lengths, refs, page), _groups(pools, refs), parents.numel(), _stream(stream, refs)
    done, scratch = _result(_scratch(n, torch.int32, refs, stream), stream), _scratch(refs.numel() + 2 * n + 2 * table.shape[0], torch.int32, refs, stream)
    _run(_library().ivftq_kv_fork_pools, refs, state, *records, _ints(parents, "parents", refs), _ints(children, "children", refs, n), n, done.data_ptr(),
         scratch.data_ptr(), where)
    return done


def kv_free(table, lengths, refs, rows, stream=None):
    """Rows give their pages back and become empty."""
    _run(_library().ivftq_kv_free, refs, _pages(table, lengths, refs, 16), _ints(rows, "rows", refs), rows.numel(), _stream(stream, refs))


def kv_trim(table, lengths, refs, page, window, sinks=0, stream=None):
    """Every row gives back the pages that no later token sees with this window and these first tokens."""
    _run(_library().ivftq_kv_trim, refs, _pages(table, lengths, refs, page), window, sinks, _stream(stream, refs))


def kv_compact(pools, table, refs, stream=None):
    """Pages in use move to the lowest numbers, in every layer of pools (several such tensors: a list of them); returns how many there
    are (device, int32 [1])."""
    state, records, where = _pages(table, None, refs, 16), _groups(pools, refs), _stream(stream, refs)
    used, scratch = _result(_scratch(1, torch.int32, refs, stream), stream), _scratch(3 * refs.numel() + 64, torch.int32, refs, stream)
    _run(_library().ivftq_kv_compact_pools, refs, state, *records, used.data_ptr(), scratch.data_ptr(), where)
    return used


def kv_copy(pools, src, dst, stream=None):
    """Record of page src[i] to page dst[i] in every layer of pools; no page both source and destination."""
    records = _pools(pools, pools)
    _run(_library().ivftq_kv_copy, pools, records, _ints(src, "src", pools), _ints(dst, "dst", pools, src.numel()), src.numel(), _stream(stream, pools))


# ---- a model's cache -----------------------------------------------------------------------------


class KVCache:
    """Keys and values of a model's layers for up to `sequences` rows of up to `tokens` tokens, in a pool of `pages` pages that all
    layers number alike.  codes=True keeps them in the 4-bit codes of the library's quantiser: `rotation_seed` and d fix the
    codec, nothing is trained.  Tensors: pools [layers, pages, ...], table, lengths, refs; methods carry the C names minus the
    prefix and queue their work on the current stream (or `stream`).

    A step of a model: `reserve` room for the new tokens, then for every layer `append` its keys and values and `attend`.  Rows
    without new tokens have none between their `starts`.  A row whose reservation was refused keeps its tokens: `append` leaves it
    out until a `reserve` grants it what it asks for, and what `attend` gives for its new rows means nothing.  lengths are not to be
    lowered by hand (a row is emptied by `free`).

    digests=True keeps a digest beside every page: `append` brings them up to date, `select` chooses each row's pages by them, and `attend`
    with those pages reads nothing else, which is what a long cache is read with."""

    def __init__(self, layers: int, heads: int, d: int, pages: int, sequences: int, tokens: int, page: int = 64, dtype=torch.bfloat16, codes: bool = False,
                 rotation_seed: int = 0, device="cuda", digests: bool = False):
        if kv_page_bytes(CODE4 if codes else _TYPES.get(dtype, -1), page, heads, d) == 0:
            raise ValueError(f"no cache of pages of {page} tokens, {heads} heads and {d} coordinates in {'codes' if codes else dtype}")
        if layers < 1 or pages < 1 or sequences < 1 or tokens < 1:
            raise ValueError("a cache has at least one layer, page, sequence and token")
        self.d, self.heads, self.page, self.codes = d, heads, page, codes
        record = (heads, page * (d + 4)) if codes else (heads, 2, page, d)
        self.pools = torch.empty((layers, pages, *record), dtype=torch.uint8 if codes else dtype, device=device)
        self.digests = torch.empty((layers, pages, heads, 2, d), dtype=torch.float16 if codes else dtype, device=device) if digests else None
        self.table = torch.full((sequences, -(-tokens // page)), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)
        self.refs = torch.zeros(pages, dtype=torch.int32, device=device)
        self._asked, self._granted = (torch.zeros(sequences, dtype=torch.int32, device=device) for _ in range(2))      # of the last reserve
        self._codec = {}
        if codes:
            self._codec = {"rotation": torch.from_numpy(ivftq_haar_rotation(d, rotation_seed)).to(device), "levels": ivftq_build_codebook(4, d)[0]}

    def reserve(self, counts, stream=None):
        granted = kv_reserve(self.table, self.lengths, self.refs, counts, self.page, stream)
        with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
            self._asked.copy_(counts)
            self._granted.copy_(granted)
        return granted

    def append(self, layer: int, k, v, starts=None, stream=None):
        kv_append(self.pools[layer], k, v, self.table, self.lengths, starts, stream=stream, asked=self._asked, granted=self._granted, **self._codec)
        if self.digests is not None:
            kv_digest(self.pools[layer], self.digests[layer], self.table, self.lengths, starts, stream=stream, asked=self._asked, granted=self._granted, **self._codec)

    def select(self, layer: int, q, count: int, starts=None, max_new: int | None = None, first: int = 1, last: int = 1, stream=None):
        """The `count` pages of each row and key-value head, for `attend`."""
        if self.digests is None:
            raise ValueError("pages are chosen by their digests: make the cache with digests=True")
        scores = kv_score(q, self.digests[layer], self.pools[layer], self.table, self.lengths, starts, max_new, stream=stream, **self._codec)
        return kv_select(scores, self.lengths, self.page, count, starts, first, last, stream=stream)

    def attend(self, layer: int, q, starts=None, max_new: int | None = None, window: int = 0, sinks: int = 0, scale=None, out=None, lse=None, stream=None, pages=None):
        if pages is not None:
            if window:
                raise ValueError("attention over chosen pages has no window: the pages say what is seen")
            return kv_attend_pages(q, self.pools[layer], self.table, self.lengths, pages, starts, max_new, scale, out=out, lse=lse, stream=stream, **self._codec)
        return kv_attend(q, self.pools[layer], self.table, self.lengths, starts, max_new, window, sinks, scale, out=out, lse=lse, stream=stream, **self._codec)

    def read(self, layer: int, k_out, v_out, starts=None, stream=None):
        kv_read(self.pools[layer], self.table, self.lengths, k_out, v_out, starts, stream=stream, **self._codec)

    def _records(self):
        return self.pools if self.digests is None else [self.pools, self.digests]

    def fork(self, parents, children, stream=None):
        return kv_fork(self._records(), self.table, self.lengths, self.refs, parents, children, self.page, stream)

    def free(self, rows, stream=None):
        kv_free(self.table, self.lengths, self.refs, rows, stream)

    def trim(self, window: int, sinks: int = 0, stream=None):
        kv_trim(self.table, self.lengths, self.refs, self.page, window, sinks, stream)

    def compact(self, stream=None):
        return kv_compact(self._records(), self.table, self.refs, stream)
