"""The calls on chosen pages without a GPU: what the host can see to be wrong is refused before anything is launched, and memory, streams and
devices are the cache's calls' own (the pointers here point nowhere that a kernel could read)."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

import paper_2605_17415_amd as pkg  # noqa: E402
from paper_2605_17415_amd import kv  # noqa: E402
from test_host_kv import BAD_CACHES, BAD_ROWS, HERE, cache, lib, pools, rows, state  # noqa: E402,F401
from test_host_kv_streams import side, world  # noqa: E402,F401

UNEVEN = C.c_void_p((1 << 20) + 8)


def queries(**changes):
    return rows(**{**dict(heads=16, row_stride=16 * 128), **changes})


def digest(lib, c=None, box=HERE, starts=None):
    return lib.ivftq_kv_digest(C.byref(c or cache()), box, starts, None)


def score(lib, c=None, q=None, box=HERE, out=HERE, starts=None, max_new=1, work=HERE, size=1 << 40):
    return lib.ivftq_kv_score(C.byref(c or cache()), C.byref(q or queries()), box, out, starts, max_new, work, size, None)


def select(lib, **changes):
    a = dict(scores=HERE, lengths=HERE, starts=None, rows=2, batch=2, heads=8, columns=4, page=64, count=8, first=1, last=1, chosen=HERE, stream=None)
    a.update(changes)
    return lib.ivftq_kv_select(*a.values())


def attend(lib, c=None, q=None, out=None, chosen=HERE, count=8, starts=None, max_new=1, scale=1.0, work=HERE, size=1 << 40):
    elsewhere = dict(data=C.c_void_p(1 << 24))
    return lib.ivftq_kv_attend_pages(C.byref(c or cache()), C.byref(q or queries()), C.byref(out or queries(**elsewhere)), None, starts, max_new, chosen, count, scale, work,
                                     size, None)


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_caches_that_are_refused(lib, change, status):
    assert [f(lib, cache(**change)) for f in (digest, score, attend)] == [status] * 3
    assert lib.ivftq_kv_score_workspace(C.byref(cache(**change)), 2, 16, 1) == -1
    assert lib.ivftq_kv_attend_pages_workspace(C.byref(cache(**change)), 2, 16, 1, 8) == -1


@pytest.mark.parametrize("change", BAD_ROWS)
def test_rows_that_are_refused(lib, change):
    q = {**change, **({"heads": 7} if "heads" in change else {})}
    assert score(lib, q=queries(**q)) == 1
    assert attend(lib, q=queries(**q)) == 1
    assert attend(lib, out=queries(**q)) == 1


def test_digests_that_are_refused(lib):
    assert digest(lib, box=None) == digest(lib, box=UNEVEN) == 1
    assert digest(lib, cache(asked=HERE)) == digest(lib, cache(granted=HERE)) == 1
    assert digest(lib, cache(batch=0)) == 0


def test_scores_that_are_refused(lib):
    assert score(lib, box=None) == score(lib, box=UNEVEN) == score(lib, out=None) == score(lib, max_new=0) == 1
    assert score(lib, work=None) == score(lib, size=100) == score(lib, work=UNEVEN) == 1
    need = lib.ivftq_kv_score_workspace(C.byref(cache()), 2, 16, 1)
    assert need >= 2 * 16 * 128 * 4 + 2 * 16 * 4 and need % 256 == 0 and score(lib, size=need - 1) == 1
    assert lib.ivftq_kv_score_workspace(C.byref(cache(format=kv.BF16)), 2, 16, 1) == 0
    assert score(lib, cache(format=kv.BF16), starts=HERE, max_new=2, size=lib.ivftq_kv_score_workspace(C.byref(cache(format=kv.BF16)), 2, 16, 2) - 1) == 1
    for bad in ((-1, 16, 1), (2, 0, 1), (2, 12, 1), (1 << 30, 16, 1), (2, 16, 0)):
        assert lib.ivftq_kv_score_workspace(C.byref(cache()), *bad) == -1
    assert score(lib, cache(batch=1 << 20, heads=1024), queries(rows=1 << 20, heads=1024, row_stride=1 << 17), starts=HERE, max_new=1 << 20) != 0
    assert score(lib, cache(batch=0), queries(rows=0)) == 0


@pytest.mark.parametrize("change,status", [(dict(page=48), 6), (dict(page=8), 6), (dict(heads=0), 6), (dict(heads=2000), 6), (dict(batch=-1), 1), (dict(columns=0), 1),
                                           (dict(columns=1 << 21), 1), (dict(rows=-1), 1), (dict(rows=1 << 30), 1), (dict(rows=3), 1), (dict(count=0), 6), (dict(count=4097), 6),
                                           (dict(first=-1), 1), (dict(last=-1), 1), (dict(first=5, last=4), 1), (dict(first=1 << 30, last=1 << 30), 1), (dict(scores=None), 1),
                                           (dict(lengths=None), 1), (dict(chosen=None), 1), (dict(chosen=C.c_void_p((1 << 20) + 2)), 1)])
def test_choices_that_are_refused(lib, change, status):
    assert select(lib, **change) == status


def test_nothing_to_choose(lib):
    assert select(lib, rows=0, batch=0, scores=None, chosen=None, lengths=None) == 0


def test_attention_that_is_refused(lib):
    assert attend(lib, chosen=None) == attend(lib, chosen=C.c_void_p((1 << 20) + 2)) == attend(lib, max_new=0) == 1
    assert attend(lib, count=0) == attend(lib, count=4097) == 6
    assert attend(lib, scale=float("nan")) == attend(lib, scale=float("inf")) == 1
    assert attend(lib, out=queries(data=C.c_void_p(1 << 24), rows=3), starts=HERE) == attend(lib, out=queries(data=C.c_void_p(1 << 24), type=kv.F16)) == 1
    assert attend(lib, cache(format=kv.BF16), out=queries()) == 1                       # results in the queries' place
    need = lib.ivftq_kv_attend_pages_workspace(C.byref(cache()), 2, 16, 1, 8)
    assert need > 0 and attend(lib, size=need - 1) == attend(lib, work=None) == attend(lib, work=UNEVEN) == 1
    for bad in ((-1, 16, 1, 8), (2, 12, 1, 8), (2, 16, 0, 8), (2, 16, 1, 0), (2, 16, 1, 4097)):
        assert lib.ivftq_kv_attend_pages_workspace(C.byref(cache()), *bad) == -1
    assert attend(lib, cache(batch=0), queries(rows=0), queries(rows=0)) == 0


def test_several_arrays_of_records(lib):
    two = (kv._Pools * 2)(pools(), pools(page_bytes=64))
    bad = (kv._Pools * 2)(pools(), pools(pages=11))
    for groups, what, status in ((0, two, 1), (9, two, 1), (2, bad, 1), (2, None, 1)):
        assert lib.ivftq_kv_fork_pools(C.byref(state()), what, groups, HERE, HERE, 1, HERE, HERE, None) == status
        assert lib.ivftq_kv_compact_pools(C.byref(state()), what, groups, HERE, HERE, None) == status
    assert lib.ivftq_kv_fork_pools(C.byref(state()), two, 2, HERE, HERE, 0, HERE, HERE, None) == 0
    assert lib.ivftq_kv_compact_pools(C.byref(state()), two, 2, None, HERE, None) == 1


def calls(w, device=0):
    """Every call, and how many tensors it gives back."""
    def t(*shape, dtype=torch.int32):
        return w.tensor(*shape, dtype=dtype, device=device)
    pool, q, box = t(4, 2, 2, 16, 64, dtype=torch.float16), t(3, 2, 64, dtype=torch.float16), t(4, 2, 2, 64, dtype=torch.float16)
    codes, rotation, half = t(4, 2, 16 * 68, dtype=torch.uint8), t(64, 64, dtype=torch.float32), t(4, 2, 2, 64, dtype=torch.float16)
    table, lengths, refs, ids, chosen = t(3, 4), t(3), t(4), t(3), t(3, 2, 5)
    scores, records = t(3, 2, 4, dtype=torch.float32), [t(1, 4, 16, dtype=torch.uint8), t(1, 4, 32, dtype=torch.uint8)]
    levels = [0.0] * 16
    return {
        "digest": (lambda **s: pkg.kv_digest(pool, box, table, lengths, **s), 0),
        "score": (lambda **s: pkg.kv_score(q, box, pool, table, lengths, **s), 1),
        "score codes": (lambda **s: pkg.kv_score(q, half, codes, table, lengths, rotation=rotation, levels=levels, **s), 1),
        "select": (lambda **s: pkg.kv_select(scores, lengths, 16, 2, **s), 1),
        "attend": (lambda **s: pkg.kv_attend_pages(q, pool, table, lengths, chosen, **s), 1),
        "fork": (lambda **s: pkg.kv_fork(records, table, lengths, refs, ids, ids, 16, **s), 1),
        "compact": (lambda **s: pkg.kv_compact(records, table, refs, **s), 1),
    }


ALL = ("digest", "score", "score codes", "select", "attend", "fork", "compact")


@pytest.mark.parametrize("name", ALL)
def test_memory_is_taken_for_the_stream_that_uses_it(world, name):  # noqa: F811
    call, results = calls(world)[name]
    s = side()
    call(stream=s)
    assert [x[2] for x in world.launched] == [77]
    assert all(stream is s for _, stream in world.allocated), world.allocated
    assert len(world.allocated) >= results and world.recorded == ["caller"] * results and world.stream == "caller"


@pytest.mark.parametrize("name", ALL)
def test_the_current_stream_and_another_device(world, name):  # noqa: F811
    calls(world)[name][0]()
    assert [x[1:] for x in world.launched] == [(0, 1000)] and not world.recorded
    world.launched.clear()
    call, _ = calls(world, device=1)[name]
    call()
    call(stream=side(1))
    assert [x[1:] for x in world.launched] == [(1, 1001), (1, 77)] and (world.device, world.stream) == (0, "caller")
    with pytest.raises(ValueError):
        call(stream=side(0))


@pytest.mark.parametrize("which", ("q", "pool", "digests", "out", "scores", "lse"))
def test_a_gradient_that_would_be_lost_is_refused(world, which):  # noqa: F811
    t = world.tensor
    pool, q, box = t(4, 2, 2, 16, 64, dtype=torch.float16), t(3, 2, 64, dtype=torch.float16), t(4, 2, 2, 64, dtype=torch.float16)
    table, lengths, chosen, scores, lse = t(3, 4), t(3), t(3, 2, 5), t(3, 2, 4, dtype=torch.float32), t(3, 2, dtype=torch.float32)
    out = t(3, 2, 64, dtype=torch.float16)
    {"q": q, "pool": pool, "digests": box, "out": out, "scores": scores, "lse": lse}[which].requires_grad_()

    def call():
        if which == "digests":
            pkg.kv_digest(pool, box, table, lengths)
        elif which == "scores":
            pkg.kv_select(scores, lengths, 16, 2)
        else:
            pkg.kv_attend_pages(q, pool, table, lengths, chosen, out=out, lse=lse)

    with pytest.raises(ValueError, match="gradient"):
        call()
    assert not world.launched
    with torch.no_grad():
        call()
    assert len(world.launched) == 1


def test_tensors_that_are_refused(world):  # noqa: F811
    t = world.tensor
    pool, q, box = t(4, 2, 2, 16, 64, dtype=torch.float16), t(3, 2, 64, dtype=torch.float16), t(4, 2, 2, 64, dtype=torch.float16)
    table, lengths, chosen, scores = t(3, 4), t(3), t(3, 2, 5), t(3, 2, 4, dtype=torch.float32)
    for bad in (t(4, 2, 2, 64, dtype=torch.bfloat16), t(5, 2, 2, 64, dtype=torch.float16), t(4, 1, 2, 64, dtype=torch.float16), t(4, 2, 2, 128, dtype=torch.float16)[..., ::2]):
        with pytest.raises(ValueError):
            pkg.kv_digest(pool, bad, table, lengths)
        with pytest.raises(ValueError):
            pkg.kv_score(q, bad, pool, table, lengths)
    for bad in (t(3, 2, 5, dtype=torch.int64), t(2, 2, 5), t(3, 1, 5), t(3, 10), t(3, 2, 10)[..., ::2]):
        with pytest.raises(ValueError):
            pkg.kv_attend_pages(q, pool, table, lengths, bad)
    for bad in (t(3, 2, 4, dtype=torch.float16), t(3, 8, dtype=torch.float32), t(3, 2, 8, dtype=torch.float32)[..., ::2]):
        with pytest.raises(ValueError):
            pkg.kv_select(bad, lengths, 16, 2)
    for bad in (t(3, 2, 3), t(3, 2, 2, dtype=torch.int64)):
        with pytest.raises(ValueError):
            pkg.kv_select(scores, lengths, 16, 2, out=bad)
    for bad in (t(3, 2, 5, dtype=torch.float32), t(3, 2, 4, dtype=torch.float64)):
        with pytest.raises(ValueError):
            pkg.kv_score(q, box, pool, table, lengths, out=bad)
    with pytest.raises(ValueError):
        pkg.kv_attend_pages(q, pool, table, lengths, chosen, out=t(3, 4, 64, dtype=torch.float16))
    assert not world.launched
