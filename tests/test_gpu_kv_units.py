"""Attention over chosen pages where neighbouring rows are worked on together (sizes: kv_units_cases.py), against float64: every format and group that
forms units, sequences that begin inside one, lists with holes and of any content, missing pages, values that are no finite numbers."""
import copy

import numpy as np
import pytest

import kv_pick_reference as pick
import kv_reference as ref
import kv_units_cases as cases

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FORMS = [("f16", "f16"), ("bf16", "bf16"), ("code4", "bf16"), ("code4", "f16")]


class Kept(ref.Cache):
    """A cache whose content in float64 is worked out once."""

    def __init__(self, *args, **more):
        super().__init__(*args, **more)
        self.full, self.seen = list(self.lens), {}

    def _kept(self, what, make, kind, b, h, n):
        key = what, kind, b, h
        if key not in self.seen:
            self.seen[key] = make(kind, b, h, self.full[b])
        return self.seen[key][:n]

    def rotated(self, kind, b, h, n):
        return self._kept("rotated", super().rotated, kind, b, h, n)

    def rows(self, kind, b, h, n):
        return self._kept("rows", super().rows, kind, b, h, n)


def _pkg():
    import paper_2605_17415_amd as pkg
    return pkg


def starts_of(news, first=0):
    return torch.tensor(first + np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32, device=DEV)


def queries(seed, rows, heads, d, dtype):
    return (torch.randn(rows, heads, d, generator=torch.Generator().manual_seed(seed)) * 1.5).to(dtype).to(DEV)


def alike(case, seed):
    """Lists of neighbours that choose much alike: pages in common, pages of one's own, holes, some of them empty."""
    rng = np.random.default_rng(seed)
    out = np.full((sum(case.news), case.heads, case.count), -1, np.int32)
    r = 0
    for n, m in zip(case.lens, case.news):
        for i in range(m):
            for h in range(case.heads):
                own = {0, (n - m + i) // 16, int(rng.integers(0, case.columns)), int(rng.integers(0, case.columns)), 3 + (i + h) // 7, 20 + i % 3}
                own = sorted(c for c in own if 0 <= c < case.columns)[: case.count]
                out[r, h, : len(own)] = own if rng.random() > 0.05 else -1
            r += 1
    return out


def blocks(case, size=6):
    """(sequence, first, past) of the rows that are compared: a sequence's first, middle and last ones; all of one with more rows than tokens."""
    for b, (n, m) in enumerate(zip(case.lens, case.news)):
        if m <= 3 * size or n < m:
            if m:
                yield b, 0, m
            continue
        for i in (0, m // 2, m - size):
            yield b, i, i + size


def check(c, case, q, out, chosen, lse):
    begin = np.cumsum([0] + case.news)
    for b, i, past in blocks(case):
        part = copy.copy(c)
        part.lens = [n if x != b else n - case.news[b] + past for x, n in enumerate(c.lens)]
        rows = slice(begin[b] + i, begin[b] + past)
        news = [past - i if x == b else 0 for x in range(len(c.lens))]
        pick.check_attention(part, q[rows].cpu(), out[rows], news, chosen[rows], None if lse is None else lse[rows])


def run(c, case, q, chosen, pool=None, **more):
    t, codec = c.device()
    lse = torch.full(q.shape[:2], 5.0, device=DEV)
    out = _pkg().kv_attend_pages(q, t["pool"] if pool is None else pool, t["table"], t["lengths"], torch.from_numpy(chosen).to(DEV), lse=lse, starts=starts_of(case.news),
                                 max_new=max(case.news), **more, **codec)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("d,page", [(64, 16), (96, 32), (128, 64), (128, 16), (192, 32), (256, 16)])
@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("group", (1, 2, 4, 5))
def test_neighbours(form, kind, d, page, group):
    case = cases.MIXED
    c = Kept(d + group, form, case.heads, d, page, case.lens, columns=case.columns)
    c.table[0, 3], c.table[2, 4] = -1, c.pages + 5                 # pages that are not there, in lists of neighbours
    q = queries(d, sum(case.news), case.heads * group, d, ref.TYPES[kind])
    chosen = alike(case, d + group)
    print(f"units {form} {kind} d={d} page={page} group={group}", flush=True)
    out, lse = run(c, case, q, chosen)
    check(c, case, q, out, chosen, lse)


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("group", (1, 4))
def test_lists_of_any_content(form, kind, group):
    """Repeats, order that falls, numbers out of range: each row passes over its own."""
    case = cases.MIXED
    c = Kept(group, form, case.heads, 64, 16, case.lens, columns=case.columns)
    odd = np.array([[3, 3, 2, 7, 7, 5, 6, 8, -9], [-5, 18, 18, 18, 2, 3, 1 << 30, -(1 << 31), 40], [40, 5, 6, 5, 6, 0, 1, 2, 41], [0, 0, 0, 1, 2, 18, 17, 16, 47],
                    [48, 1, 2, 3, 4, 5, 6, 7, 8], [-1, 4, -1, 9, -1, 11, -1, 47, 47], [-1] * 9], np.int32)
    rows = sum(case.news)
    chosen = odd[np.random.default_rng(group).integers(0, len(odd), (rows, case.heads))].copy()
    q = queries(1, rows, case.heads * group, 64, ref.TYPES[kind])
    out, lse = run(c, case, q, chosen)
    check(c, case, q, out, chosen, lse)


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("d,page", [(64, 32), (128, 16), (256, 64)])
@pytest.mark.parametrize("group", (1, 2, 5))
def test_no_numbers_in_a_neighbours_page(form, kind, d, page, group):
    """What one row has chosen may be anything to the others of its unit; they keep their results to the last bit."""
    n, new, mine = 9 * page, 260, (3, 130, 259)
    case = cases.Case(heads=4, lens=[n + new], news=[new], columns=-(-(n + new) // page), count=5)
    c = Kept(7, form, 4, d, page, case.lens, spare=2)
    q = queries(7, new, 4 * group, d, ref.TYPES[kind])
    chosen = np.full((new, 4, 5), -1, np.int32)
    for r in range(new):
        chosen[r, :, :4] = [0, 2 + r % 3, 5, 8]
    chosen[list(mine)] = [0, 1, 2, 7, 8]                           # pages 1 and 7 are these rows' alone, page 6 is nobody's
    want, sums = run(c, case, q, chosen)
    check(c, case, q, want, chosen, sums)
    others = [r for r in range(new) if r not in mine]
    t, _ = c.device()
    for col in (1, 6, 7):
        t["pool"][int(c.table[0, col])] = 255 if form == "code4" else torch.nan
    got, lse = run(c, case, q, chosen, t["pool"])
    assert torch.equal(got[others], want[others]) and torch.equal(lse[others], sums[others]) and torch.isnan(got[list(mine)].float()).any(-1).all()
    if form == "code4":
        return
    clean, _ = c.device()                                          # infinite values, keys as they were
    clean["pool"][int(c.table[0, 7]), :, 1] = torch.inf
    got, lse = run(c, case, q, chosen, clean["pool"])
    assert torch.equal(got[others], want[others]) and torch.equal(lse, sums) and (got[list(mine)] == torch.inf).all()
    clean, _ = c.device()                                          # one value of one head, and every row of the unit sees tokens of the page before it
    clean["pool"][int(c.table[0, 7]), 2, 1].view(page // 8, d, 8)[0, d - 1, 3] = -torch.inf
    got, lse = run(c, case, q, chosen, clean["pool"])
    assert torch.equal(got[others], want[others]) and torch.equal(lse, sums)
    heads = slice(2 * group, 3 * group)
    assert (got[list(mine), heads, d - 1] == -torch.inf).all()
    got[list(mine), heads, d - 1] = want[list(mine), heads, d - 1]
    # (such a token is added by itself, in float32 and with its weight not rounded: the row's other coordinates as they may be off)
    check(c, case, q, got, chosen, lse)


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("group", (1, 3))
def test_rows_that_keep_what_they_have(form, kind, group):
    """Queries and results inside wider rows, rows of no sequence before and behind the others, rows past max_new."""
    case, most = cases.PARTS, 50
    rows, first = sum(case.news), 7
    heads = case.heads * group
    c = Kept(8, form, case.heads, 64, 16, case.lens, columns=case.columns)
    wide = queries(8, rows + 20, heads + 6, 64, ref.TYPES[kind])
    place = torch.full((rows + 20, heads + 5, 64), 3.0, dtype=wide.dtype, device=DEV)
    chosen = alike(case, group)
    every = np.concatenate([chosen[:first], chosen, chosen[: 20 - first]])
    t, codec = c.device()
    lse = torch.full((rows + 20, heads), 5.0, device=DEV)
    _pkg().kv_attend_pages(wide[:, 3: 3 + heads], t["pool"], t["table"], t["lengths"], torch.from_numpy(every).to(DEV), starts=starts_of(case.news, first), max_new=most,
                           out=place[:, 2: 2 + heads], lse=lse, **codec)
    assert (place[:, :2] == 3).all() and (place[:, 2 + heads:] == 3).all()
    begin = first + np.cumsum([0] + case.news)
    done = np.concatenate([np.arange(a, a + min(m, most)) for a, m in zip(begin, case.news)])
    kept = [r for r in range(rows + 20) if r not in set(done.tolist())]
    assert (place[kept] == 3).all() and (lse[kept] == 5).all()
    part = cases.Case(case.heads, [n - max(m - most, 0) for n, m in zip(case.lens, case.news)], [min(m, most) for m in case.news], case.columns, case.count)
    c.lens = part.lens
    check(c, part, wide[done][:, 3: 3 + heads], place[done][:, 2: 2 + heads], every[done], lse[done])


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("scale", (0.0, -0.2))
def test_scales(form, kind, scale):
    case = cases.MIXED
    c = Kept(4, form, case.heads, 64, 16, case.lens, columns=case.columns)
    q = queries(4, sum(case.news), case.heads * 2, 64, ref.TYPES[kind])
    chosen = alike(case, 4)
    out, _ = run(c, case, q, chosen, scale=scale)
    begin = np.cumsum([0] + case.news)
    for b, i, past in blocks(case):
        part = copy.copy(c)
        part.lens = [n if x != b else n - case.news[b] + past for x, n in enumerate(c.lens)]
        rows = slice(begin[b] + i, begin[b] + past)
        pick.check_attention(part, q[rows].cpu(), out[rows], [past - i if x == b else 0 for x in range(len(c.lens))], chosen[rows], scale=scale)


def test_long_lists():
    """Of so many pages that two rows fit a unit."""
    case = cases.LONG_LISTS
    c = Kept(3, "bf16", case.heads, 64, 16, case.lens, columns=case.columns)
    q = queries(3, sum(case.news), case.heads, 64, torch.bfloat16)
    rng = np.random.default_rng(3)
    chosen = np.sort(np.stack([rng.permutation(case.columns)[: case.count] for _ in range(sum(case.news) * case.heads)]), axis=1)
    chosen = chosen.astype(np.int32).reshape(-1, case.heads, case.count)
    out, lse = run(c, case, q, chosen)
    check(c, case, q, out, chosen, lse)


def test_wide_tables():
    """Columns past 2^13, so that the bits of eight rows fit a unit; the table names few pages over and over."""
    case = cases.WIDE_TABLE
    c = Kept(5, "bf16", case.heads, 64, 16, [320], columns=case.columns, spare=0)
    c.lens = c.full = list(case.lens)
    c.table[0] = np.random.default_rng(5).integers(0, c.pages, case.columns)
    q = queries(5, sum(case.news), case.heads, 64, torch.bfloat16)
    rng = np.random.default_rng(6)
    chosen = np.sort(rng.integers(0, case.columns, (sum(case.news), case.heads, case.count)).astype(np.int32), axis=2)
    chosen[:, :, -3:] = case.columns - 40 + np.arange(3) * 17      # some in common; a repeat among the others is passed over
    chosen.sort(axis=2)
    out, lse = run(c, case, q, chosen)
    check(c, case, q, out, chosen, lse)
