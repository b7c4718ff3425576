"""A step whose reservation was refused for some rows: their new tokens have no place, and what their pages hold stays."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _pkg():
    import paper_2605_17415_amd as pkg
    return pkg


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def rows(seed, n, heads=2, d=64):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [torch.randn(n, heads, d, generator=g, device=DEV).bfloat16() for _ in range(2)]


def content(cache, row, n):
    """The first n tokens' keys and values of a row."""
    k, v = (torch.full((n, cache.heads, cache.d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    _pkg().kv_read(cache.pools[0], cache.table[row:row + 1], ints([n]), k, v, starts=ints([0, n]), **cache._codec)
    return torch.stack([k, v])


@pytest.mark.parametrize("codes", (False, True))
@pytest.mark.parametrize("many", (False, True))
@pytest.mark.parametrize("sequences", (4, 70))
def test_a_refused_row_keeps_its_tokens(codes, many, sequences):
    """Rows 0 and 1 share full pages; row 0 asks for more than there is, row 2 is served."""
    cache = _pkg().KVCache(1, 2, 64, pages=8, sequences=sequences, tokens=400, page=16, codes=codes, device=DEV)
    rest = [0] * (sequences - 4)
    assert cache.reserve(ints([32, 0, 5, 0] + rest)).tolist() == [32, 0, 5, 0] + rest
    k, v = rows(1, 37)
    cache.append(0, k, v, ints([0, 32, 32, 37, 37] + [37] * len(rest)))
    assert cache.fork(ints([0]), ints([1])).tolist() == [1]
    before = content(cache, 0, 32), content(cache, 2, 5)
    if many:
        news = [100, 0, 3, 200] + rest
        got = [0, 0, 3, 0] + rest
        starts = ints([0, 100, 100, 103, 303] + [303] * len(rest))
        fresh = [x[100:103] for x in rows(2, 303)]
    else:
        # one row a sequence: the pages are taken first, so that a row at a page's end gets none
        assert cache.reserve(ints([0, 0, 0, 80] + rest)).tolist() == [0, 0, 0, 80] + rest
        news = [1, 1, 1, 0] + rest
        got = [0, 0, 1, 0] + rest
        starts = None
        fresh = [x[2:3] for x in rows(2, sequences)]
    counts = ints(news)
    assert cache.reserve(counts).tolist() == got
    counts.fill_(0)                                         # the caller's own again
    cache.append(0, *rows(2, 303 if many else sequences), starts)
    assert torch.equal(content(cache, 0, 32), before[0]) and torch.equal(content(cache, 1, 32), before[0])
    n = 5 + got[2]
    now = content(cache, 2, n)
    assert torch.equal(now[:, :5], before[1])
    if not codes:
        assert torch.equal(now[0, 5:], fresh[0]) and torch.equal(now[1, 5:], fresh[1])
    else:
        assert all((now[i, 5:] - x).float().norm() < 0.2 * x.float().norm() for i, x in enumerate(fresh))
    # room is made and the reservation repeated: now they are written
    cache.free(ints([3]))
    cache.reserve(ints([16, 0, 0, 0] + rest))
    k, v = rows(3, 16)
    cache.append(0, k, v, ints([0, 16, 16, 16, 16] + [16] * len(rest)))
    now = content(cache, 0, 48)
    assert torch.equal(now[:, :32], before[0]) and torch.equal(content(cache, 1, 32), before[0])
    assert (now[0, 32:] - k).float().norm() < 0.2 * k.float().norm()


def test_with_the_calls_themselves():
    """asked and granted as kv_reserve has them; without them every row is written."""
    pkg = _pkg()
    pool = torch.zeros(4, 2, 2, 16, 64, dtype=torch.bfloat16, device=DEV)
    table, lengths = ints([0, 1, 2, 3]).view(4, 1), ints([3, 9, 16, 1])
    k, v = rows(4, 4)
    pkg.kv_append(pool, k, v, table, lengths, asked=ints([1, 1, 1, -5]), granted=ints([1, 0, 1, 0]))
    written = pool.abs().sum((1, 2, 3, 4)) > 0
    assert written.tolist() == [True, False, True, True]
    pkg.kv_append(pool, k, v, table, lengths)
    assert torch.equal(pool[1, :, 0, 8], k[1])
    for one in (dict(asked=ints([1] * 4)), dict(granted=ints([1] * 4)), dict(asked=ints([1] * 3), granted=ints([1] * 4)), dict(asked=ints([1] * 4).long(), granted=ints([1] * 4))):
        with pytest.raises((TypeError, ValueError, pkg.IvftqError)):
            pkg.kv_append(pool, k, v, table, lengths, **one)


@pytest.mark.parametrize("codes", (False, True))
def test_a_recorded_step_leaves_refused_rows_out(codes):
    """Reserve, append and attend recorded once; replayed until the pages run out and past that, with eager reads between."""
    cache = _pkg().KVCache(1, 2, 64, pages=3, sequences=2, tokens=400, page=16, codes=codes, device=DEV)
    cache.reserve(ints([14, 15]))
    k, v = rows(1, 29)
    starts = ints([0, 14, 29])
    cache.append(0, k, v, starts)
    one, two = rows(2, 2)
    q, counts, out = torch.randn(2, 4, 64, device=DEV).bfloat16(), ints([1, 1]), torch.empty(2, 4, 64, dtype=torch.bfloat16, device=DEV)

    def step():
        granted = cache.reserve(counts)
        cache.append(0, one, two)
        cache.attend(0, q, out=out)
        return granted

    state = [x.clone() for x in (cache.table, cache.lengths, cache.refs, cache.pools)]
    step()                                                  # (what a first call sets up is not recorded)
    for x, y in zip((cache.table, cache.lengths, cache.refs, cache.pools), state):
        x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        granted = step()
    lengths = [14, 15]
    for n in range(8):                                      # row 1 takes the third page for its 17th token, row 0 ends at its 16th
        before = [content(cache, r, lengths[r]) for r in range(2)]
        for x, seed in ((one, 10 + n), (two, 30 + n)):
            x.copy_(rows(seed, 2)[0])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = [1 if lengths[0] < 16 else 0, 1]
        assert granted.tolist() == want
        for r in range(2):
            assert torch.equal(content(cache, r, lengths[r]), before[r]), (n, r)
            lengths[r] += want[r]
            if want[r]:
                now = content(cache, r, lengths[r])[:, -1]
                assert (now[0] - one[r]).float().norm() < 0.2 * one[r].float().norm() and (now[1] - two[r]).float().norm() < 0.2 * two[r].float().norm()
        assert cache.lengths.tolist() == lengths
    assert lengths == [16, 23]
