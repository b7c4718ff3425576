"""Pages of the cache taken, shared, given back, brought together and copied, against a plain walk through the rules."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _pkg():
    import paper_2605_17415_amd as pkg
    return pkg


class Plain:
    """The rules, one page at a time."""

    def __init__(self, rows, columns, pages, page, layers=2, record=48, seed=0):
        self.page, self.columns = page, columns
        self.table = np.full((rows, columns), -1, np.int32)
        self.lengths, self.refs = np.zeros(rows, np.int32), np.zeros(pages, np.int32)
        self.pools = np.random.default_rng(seed).integers(0, 256, (layers, pages, record), dtype=np.uint8)

    def free_page(self):
        z = np.nonzero(self.refs <= 0)[0]
        return int(z[0]) if len(z) else None

    def reserve(self, counts):
        out, short = np.zeros(len(counts), np.int32), False
        for r, n in enumerate(counts):
            n = max(int(n), 0)
            have, want = -(-int(self.lengths[r]) // self.page), -(-(int(self.lengths[r]) + n) // self.page)
            if want > self.columns:
                continue
            if want > have and (short or (self.refs <= 0).sum() < want - have):
                short = True
                continue
            for c in range(have, want):
                self.table[r, c] = self.free_page()
                self.refs[self.table[r, c]] = 1
            self.lengths[r] += n
            out[r] = n
        return out

    def fork(self, parents, children):
        rows, seen, out, was = len(self.table), set(), [], self.lengths.copy()
        short = False
        for p, c in zip(parents, children):
            ok = 0 <= p < rows and 0 <= c < rows and c not in seen and c not in parents and was[c] == 0
            if 0 <= c < rows:
                seen.add(c)
            if ok and self.lengths[p] % self.page:
                new = None if short else self.free_page()
                if new is None:
                    short, ok = True, False
            if ok:
                n = int(self.lengths[p])
                self.table[c] = -1
                for j in range(n // self.page):
                    self.table[c, j] = self.table[p, j] if 0 <= self.table[p, j] < len(self.refs) else -1
                    if self.table[c, j] >= 0:
                        self.refs[self.table[c, j]] += 1
                if n % self.page:
                    self.table[c, n // self.page] = new
                    self.refs[new] = 1
                    if self.table[p, n // self.page] >= 0:
                        self.pools[:, new] = self.pools[:, self.table[p, n // self.page]]
                self.lengths[c] = n
            out.append(int(ok))
        return out

    def give(self, r, columns):
        for c in columns:
            if 0 <= self.table[r, c] < len(self.refs):
                self.refs[self.table[r, c]] -= 1
            self.table[r, c] = -1

    def free(self, rows):
        for r in rows:
            if 0 <= r < len(self.table):
                self.give(r, range(self.columns))
                self.lengths[r] = 0

    def trim(self, window, sinks):
        for r, n in enumerate(self.lengths):
            self.give(r, [c for c in range(self.columns) if (c + 1) * self.page <= n - window + 1 and c * self.page >= sinks])

    def compact(self):
        used = int((self.refs > 0).sum())
        high = [p for p in range(len(self.refs)) if self.refs[p] > 0 and p >= used]
        holes = [p for p in range(used) if self.refs[p] <= 0]
        for a, b in zip(high, holes):
            self.pools[:, b] = self.pools[:, a]
            self.refs[b], self.refs[a] = self.refs[a], 0
            self.table[self.table == a] = b
        return used


class Both:
    def __init__(self, *a, **k):
        self.p = Plain(*a, **k)
        self.table, self.lengths, self.refs, self.pools = (torch.from_numpy(x.copy()).to(DEV) for x in (self.p.table, self.p.lengths, self.p.refs, self.p.pools))

    def ints(self, x):
        return torch.tensor(list(x), dtype=torch.int32, device=DEV)

    def reserve(self, counts):
        got = _pkg().kv_reserve(self.table, self.lengths, self.refs, self.ints(counts), page=self.p.page)
        assert np.array_equal(got.cpu().numpy(), self.p.reserve(counts))
        self.same()

    def fork(self, parents, children):
        got = _pkg().kv_fork(self.pools, self.table, self.lengths, self.refs, self.ints(parents), self.ints(children), page=self.p.page)
        assert got.tolist() == self.p.fork(parents, children)
        self.same()

    def free(self, rows):
        _pkg().kv_free(self.table, self.lengths, self.refs, self.ints(rows))
        self.p.free(rows)
        self.same()

    def trim(self, window, sinks=0):
        _pkg().kv_trim(self.table, self.lengths, self.refs, page=self.p.page, window=window, sinks=sinks)
        self.p.trim(window, sinks)
        self.same()

    def compact(self):
        got = _pkg().kv_compact(self.pools, self.table, self.refs)
        assert got.tolist() == [self.p.compact()]
        self.same()

    def same(self):
        torch.cuda.synchronize()
        for a, b in ((self.table, self.p.table), (self.lengths, self.p.lengths), (self.refs, self.p.refs), (self.pools, self.p.pools)):
            assert np.array_equal(a.cpu().numpy(), b)


@pytest.mark.parametrize("page", (16, 64))
def test_a_life_of_a_cache(page):
    s = Both(12, 20, 60, page)
    s.reserve([0, 1, page, page + 1, 5 * page, -3, 7, 0, 0, 0, 0, 0])
    s.fork([3, 4, 1, 3], [0, 7, 8, 9])
    s.reserve([1] * 12)
    s.free([4, 3, 4, 99, -1])
    s.compact()
    s.reserve([3 * page] * 12)
    s.fork([0, 0, 11, 2], [5, 3, 1, 2])                     # 5, 1 and 2 are not empty; row 3 was given pages again too
    s.free(range(3, 9))
    s.trim(page + 3, sinks=1)
    s.compact()
    s.trim(1)
    s.reserve([page] * 12)
    s.free(range(12))
    assert int(s.refs.sum()) == 0
    s.compact()


def test_pages_run_out():
    s = Both(6, 8, 9, 16)
    s.reserve([16, 40, 64, 32, 0, 16])                      # 1 + 3 + 4 pages; two more do not fit, nor do later ones that need any
    s.reserve([0, 8, 0, 1, 0, 17])
    s.free([1])
    s.reserve([3, 0, 129, 33, 16, 16])                      # 129: over the columns
    s.fork([0, 3], [1, 1])
    s.fork([3, 0], [5, 0])


def test_fork_refusals():
    s = Both(8, 4, 30, 16)
    s.reserve([20, 16, 40, 0, 0, 0, 0, 0])
    s.fork([0, 0, 1, 2, -1, 0, 9, 3, 2, 4], [3, 3, 0, 4, 5, 8, 6, 7, 5, 6])      # twice, into a parent, out of range, from an empty row that is a child
    s.fork([2, 2, 2], [6, 7, 3])


def test_many_rows_and_pages():
    """More rows than threads, more pages than one pass of the scans."""
    rng = np.random.default_rng(3)
    s = Both(2500, 6, 9000, 16, layers=1, record=16)
    s.reserve(rng.integers(0, 60, 2500))
    dead = rng.choice(2500, 1300, replace=False)
    s.free(dead)
    empty = [int(r) for r in np.nonzero(s.p.lengths == 0)[0]]
    full = [int(r) for r in np.nonzero(s.p.lengths > 0)[0]]
    n = min(len(empty), len(full), 1200)
    s.fork(full[:n], empty[:n])
    s.compact()
    s.reserve(rng.integers(0, 30, 2500))
    s.free(rng.choice(2500, 2000, replace=False))
    s.compact()


@pytest.mark.parametrize("record", (16, 16_384, 16_400, 50_000))
def test_copy(record):
    pools = torch.randint(0, 256, (3, 40, record), dtype=torch.uint8, device=DEV)
    part = pools[1:]                                        # layers of a larger tensor
    want = part.clone()
    src, dst = torch.tensor([3, 3, 39, 50, -1, 7], dtype=torch.int32, device=DEV), torch.tensor([0, 1, 20, 2, 4, 40], dtype=torch.int32, device=DEV)
    want[:, 0], want[:, 1], want[:, 20] = want[:, 3].clone(), want[:, 3].clone(), want[:, 39].clone()
    first = pools[0].clone()
    _pkg().kv_copy(part, src, dst)
    torch.cuda.synchronize()
    assert torch.equal(part, want) and torch.equal(pools[0], first)


def test_in_a_graph():
    """Reserving and forking recorded once; the state is set back by eager copies between the replays."""
    s = Both(6, 8, 40, 16)
    s.reserve([20, 33, 5, 0, 0, 0])
    keep = [x.clone() for x in (s.table, s.lengths, s.refs, s.pools)]
    parents, children, counts = s.ints([0, 1]), s.ints([3, 4]), s.ints([1, 0, 30, 2, 2, 9])
    pkg = _pkg()

    def turn():
        done = pkg.kv_fork(s.pools, s.table, s.lengths, s.refs, parents, children, page=16)
        return done, pkg.kv_reserve(s.table, s.lengths, s.refs, counts, page=16)

    done, granted = turn()
    torch.cuda.synchronize()
    want = [x.clone() for x in (done, granted, s.table, s.lengths, s.refs, s.pools)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        done, granted = turn()
    for _ in range(3):
        for x, y in zip((s.table, s.lengths, s.refs, s.pools), keep):
            x.copy_(y)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((done, granted, s.table, s.lengths, s.refs, s.pools), want))
