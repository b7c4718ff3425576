"""The key-value cache's C ABI without a GPU: every declared symbol is exported and bound, and what the host can see to be wrong is
refused before anything is launched (the pointers here point nowhere that a kernel could read)."""
import ctypes as C
import os
import re

import numpy as np
import pytest

import paper_2605_17415_amd as pkg
from paper_2605_17415_amd import kv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = C.c_void_p(1 << 20)          # aligned, never followed: every call below is refused


@pytest.fixture(scope="module")
def lib():
    return kv._library()


def cache(**changes):
    levels = pkg.ivftq_build_codebook(4, 128)[0]
    fields = dict(pool=HERE, table=HERE, lengths=HERE, rotation=HERE, pages=10, table_stride=4, batch=2, columns=4, format=kv.CODE4, page=64, heads=8, d=128)
    fields.update(changes)
    if "levels" not in fields:
        fields["levels"] = (C.c_float * 16)(*levels)
    return kv._Cache(**fields)


def rows(**changes):
    fields = dict(data=HERE, row_stride=8 * 128, head_stride=128, rows=2, heads=8, type=kv.BF16)
    fields.update(changes)
    return kv._Rows(**fields)


def state(**changes):
    fields = dict(table=HERE, lengths=HERE, refs=HERE, table_stride=4, pages=10, rows=2, columns=4, page=64)
    fields.update(changes)
    return kv._Pages(**fields)


def pools(**changes):
    fields = dict(pool=HERE, layer_stride=1 << 20, page_bytes=4096, pages=10, layers=2)
    fields.update(changes)
    return kv._Pools(**fields)


def test_every_declared_symbol_is_exported_and_bound(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ivftq_kv.h")).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(ivftq_[a-z_0-9]+)\s*\(", text)))
    assert declared == sorted(pkg.declared_kv_symbols())
    for name in declared:
        assert hasattr(lib, name)


@pytest.mark.parametrize("form,per_token", [(kv.F16, 512), (kv.BF16, 512), (kv.CODE4, 132)])
def test_bytes_of_a_page(form, per_token):
    assert pkg.kv_page_bytes(form, 64, 8, 128) == 64 * 8 * per_token
    for bad in ((3, 64, 8, 128), (form, 48, 8, 128), (form, 8, 8, 128), (form, 2048, 8, 128), (form, 64, 0, 128), (form, 64, 8, 100)):
        assert pkg.kv_page_bytes(*bad) == 0


def flip(levels, i, v):
    a = np.array(levels, np.float32)
    a[i] = v
    return (C.c_float * 16)(*a)


BAD_CACHES = [(dict(format=7), 1), (dict(d=100), 6), (dict(d=0), 6), (dict(page=48), 6), (dict(page=8), 6), (dict(heads=0), 6), (dict(heads=2000), 6),
              (dict(pages=0), 1), (dict(pages=1 << 40), 1), (dict(batch=-1), 1), (dict(columns=0), 1), (dict(table_stride=3), 1), (dict(pool=None), 1),
              (dict(table=None), 1), (dict(lengths=None), 1), (dict(pool=C.c_void_p((1 << 20) + 8)), 1), (dict(rotation=None), 1),
              (dict(rotation=C.c_void_p((1 << 20) + 4)), 1), (dict(levels=(C.c_float * 16)()), 1),
              (dict(levels=flip(pkg.ivftq_build_codebook(4, 128)[0], 3, -0.07)), 1), (dict(levels=flip(pkg.ivftq_build_codebook(4, 128)[0], 15, float("nan"))), 1),
              (dict(levels=flip(pkg.ivftq_build_codebook(4, 128)[0], 15, float("inf"))), 1)]
BAD_ROWS = [dict(data=None), dict(type=2), dict(heads=7), dict(rows=3), dict(rows=-1), dict(row_stride=1023), dict(head_stride=4), dict(head_stride=120),
            dict(data=C.c_void_p((1 << 20) + 2)), dict(row_stride=-8)]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_a_bad_cache_is_refused_everywhere(lib, change, status):
    c, r = cache(**change), rows()
    assert lib.ivftq_kv_append(C.byref(c), C.byref(r), C.byref(r), None, None) == status
    assert lib.ivftq_kv_read(C.byref(c), C.byref(r), C.byref(r), None, None) == status
    assert lib.ivftq_kv_attend(C.byref(c), C.byref(r), C.byref(r), None, None, 1, 0, 0, 0.1, HERE, 1 << 40, None) == status
    assert lib.ivftq_kv_attend_workspace(C.byref(c), 2, 8, 1) == -1
    assert len(lib.ivftq_last_error()) > 5


@pytest.mark.parametrize("change", BAD_ROWS)
def test_bad_rows_are_refused(lib, change):
    c, r, good = cache(), rows(**change), rows()
    for k, v in ((r, good), (good, r)):
        assert lib.ivftq_kv_append(C.byref(c), C.byref(k), C.byref(v), None, None) == 1
        assert lib.ivftq_kv_read(C.byref(c), C.byref(k), C.byref(v), None, None) == 1
        assert lib.ivftq_kv_attend(C.byref(c), C.byref(k), C.byref(v), None, None, 1, 0, 0, 0.1, HERE, 1 << 40, None) == 1


def test_more_pieces_of_rows_than_a_launch_counts_are_refused(lib):
    """One row per sequence: 2^28 heads of 8 pieces of eight coordinates."""
    c = cache(format=kv.BF16, batch=1 << 20, heads=256, d=64, columns=1, table_stride=1)
    r = rows(row_stride=256 * 64, head_stride=64, rows=1 << 20, heads=256)
    assert lib.ivftq_kv_append(C.byref(c), C.byref(r), C.byref(r), None, None) == 6
    assert lib.ivftq_kv_read(C.byref(c), C.byref(r), C.byref(r), None, None) == 6


def test_types_of_rows_and_cache(lib):
    c = cache(format=kv.F16)
    assert lib.ivftq_kv_append(C.byref(c), C.byref(rows()), C.byref(rows()), None, None) == 1            # bfloat16 into a float16 cache
    c = cache()
    assert lib.ivftq_kv_append(C.byref(c), C.byref(rows()), C.byref(rows(type=kv.F16)), None, None) == 1    # two types


@pytest.mark.parametrize("max_new,window,sinks,scale", [(0, 0, 0, 0.1), (1, -1, 0, 0.1), (1, 0, -1, 0.1), (1, 0, 0, float("nan")), (1, 0, 0, float("inf"))])
def test_bad_masks_are_refused(lib, max_new, window, sinks, scale):
    c, r = cache(), rows()
    assert lib.ivftq_kv_attend(C.byref(c), C.byref(r), C.byref(r), None, None, max_new, window, sinks, scale, HERE, 1 << 40, None) == 1


def test_workspace_too_small_or_crooked_is_refused(lib):
    c, r = cache(), rows()
    need = lib.ivftq_kv_attend_workspace(C.byref(c), 2, 8, 1)
    assert need > 0
    for where, size in ((HERE, need - 1), (None, need), (C.c_void_p((1 << 20) + 128), need)):
        assert lib.ivftq_kv_attend(C.byref(c), C.byref(r), C.byref(r), None, None, 1, 0, 0, 0.1, where, size, None) == 1
    assert lib.ivftq_kv_attend_workspace(C.byref(c), 2, 9, 1) == -1                                       # 9 query heads over 8
    assert lib.ivftq_kv_attend_workspace(C.byref(c), -1, 8, 1) == -1


def test_nothing_to_do_is_no_error(lib):
    c, r = cache(batch=0), rows(rows=0)
    assert lib.ivftq_kv_append(C.byref(c), C.byref(r), C.byref(r), None, None) == 0
    assert lib.ivftq_kv_attend(C.byref(c), C.byref(r), C.byref(r), None, None, 1, 0, 0, 0.1, None, 0, None) == 0
    assert lib.ivftq_kv_free(C.byref(state()), None, 0, None) == 0
    assert lib.ivftq_kv_fork(C.byref(state()), C.byref(pools()), None, None, 0, None, None, None) == 0
    assert lib.ivftq_kv_copy(C.byref(pools()), None, None, 0, None) == 0
    assert lib.ivftq_kv_reserve(C.byref(state(rows=0)), HERE, HERE, HERE, None) == 0


@pytest.mark.parametrize("change", [dict(page=48), dict(pages=0), dict(rows=-1), dict(columns=0), dict(table_stride=3), dict(table=None), dict(refs=None),
                                    dict(columns=1 << 21, table_stride=1 << 21)])
def test_a_bad_state_of_pages_is_refused(lib, change):
    s = state(**change)
    assert lib.ivftq_kv_reserve(C.byref(s), HERE, HERE, HERE, None) in (1, 6)
    assert lib.ivftq_kv_fork(C.byref(s), C.byref(pools()), HERE, HERE, 1, HERE, HERE, None) in (1, 6)
    assert lib.ivftq_kv_free(C.byref(s), HERE, 1, None) in (1, 6)
    assert lib.ivftq_kv_trim(C.byref(s), 100, 0, None) in (1, 6)
    assert lib.ivftq_kv_compact(C.byref(s), C.byref(pools()), HERE, HERE, None) in (1, 6)


@pytest.mark.parametrize("change", [dict(pool=None), dict(page_bytes=0), dict(page_bytes=4100), dict(layer_stride=4096), dict(layer_stride=(1 << 20) + 8),
                                    dict(layers=0), dict(pages=0), dict(pool=C.c_void_p((1 << 20) + 8))])
def test_bad_pools_are_refused(lib, change):
    p = pools(**change)
    assert lib.ivftq_kv_copy(C.byref(p), HERE, HERE, 1, None) == 1
    assert lib.ivftq_kv_fork(C.byref(state()), C.byref(p), HERE, HERE, 1, HERE, HERE, None) == 1
    assert lib.ivftq_kv_compact(C.byref(state()), C.byref(p), HERE, HERE, None) == 1


def test_other_refusals_about_pages(lib):
    assert lib.ivftq_kv_trim(C.byref(state()), 0, 0, None) == 1
    assert lib.ivftq_kv_trim(C.byref(state()), 5, -1, None) == 1
    assert lib.ivftq_kv_free(C.byref(state()), HERE, -1, None) == 1
    assert lib.ivftq_kv_free(C.byref(state()), None, 1, None) == 1
    assert lib.ivftq_kv_copy(C.byref(pools()), HERE, None, 1, None) == 1
    assert lib.ivftq_kv_fork(C.byref(state(pages=11)), C.byref(pools()), HERE, HERE, 1, HERE, HERE, None) == 1
    assert lib.ivftq_kv_fork(C.byref(state()), C.byref(pools()), HERE, HERE, 70000, HERE, HERE, None) == 1
    assert lib.ivftq_kv_compact(C.byref(state(pages=11)), C.byref(pools()), HERE, HERE, None) == 1
    assert lib.ivftq_kv_reserve(C.byref(state()), None, HERE, HERE, None) == 1


def test_tensors_that_are_no_device_tensors_are_refused():
    torch = pytest.importorskip("torch")
    pool = torch.zeros(4, 2, 2, 16, 64, dtype=torch.float16)
    q, table, lengths = torch.zeros(1, 2, 64, dtype=torch.float16), torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        pkg.kv_attend(q, pool, table, lengths)
    with pytest.raises(TypeError):
        pkg.kv_append(pool, q, q, table, lengths)
    with pytest.raises(TypeError):
        pkg.kv_copy(pool, table, table)


@pytest.mark.parametrize("one", ("asked", "granted"))
def test_half_of_a_reservation_is_refused(lib, one):
    c, r = cache(**{one: HERE}), rows()
    assert lib.ivftq_kv_append(C.byref(c), C.byref(r), C.byref(r), None, None) == 1
    c = cache(asked=HERE, granted=C.c_void_p((1 << 20) + 2))
    assert lib.ivftq_kv_append(C.byref(c), C.byref(r), C.byref(r), None, None) == 1


def test_a_workspace_for_more_workgroups_than_a_call_takes_is_refused(lib):
    """What the call refuses, the question for its workspace refuses too: 2^20 sequences of up to 2^19 row tiles."""
    c = cache(format=kv.BF16, batch=1 << 20, heads=8, d=64)
    r = rows(rows=1 << 23, heads=64, row_stride=64 * 64, head_stride=64)
    assert lib.ivftq_kv_attend(C.byref(c), C.byref(r), C.byref(r), None, HERE, 1 << 23, 0, 0, 0.1, HERE, 1 << 40, None) == 6
    assert lib.ivftq_kv_attend_workspace(C.byref(c), 1 << 23, 64, 1 << 23) == -1
    assert b"workgroups" in lib.ivftq_last_error()


@pytest.mark.parametrize("form", (kv.F16, kv.BF16))
def test_results_over_the_queries_are_refused_in_16_bits(lib, form):
    """Other workgroups still read the queries when a result is written."""
    c, q = cache(format=form), rows(type=form)
    for columns in (4, 400):
        c.columns = c.table_stride = columns
        assert lib.ivftq_kv_attend(C.byref(c), C.byref(q), C.byref(q), None, None, 1, 0, 0, 0.1, HERE, 1 << 40, None) == 1
        assert b"out" in lib.ivftq_last_error()
