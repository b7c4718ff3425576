"""Digests of pages, their scores and the pages chosen by them against float64: every format and head size, pages that go on, rows that reach
nothing, missing pages, ties, what is no number."""
import numpy as np
import pytest

import kv_pick_reference as pick
import kv_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FORMS = [("f16", "f16"), ("bf16", "bf16"), ("code4", "bf16"), ("code4", "f16")]
SIZES = [(64, 16), (96, 32), (128, 64), (192, 16), (256, 128), (128, 1024)]


def _pkg():
    import paper_2605_17415_amd as pkg
    return pkg


def starts_of(news):
    return torch.tensor([0] + list(np.cumsum(news)), dtype=torch.int32, device=DEV)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def blank_digests(c, value=7.0):
    kind = torch.float16 if c.form == "code4" else ref.TYPES[c.form]
    return torch.full((c.pages, c.heads, 2, c.d), value, dtype=kind, device=DEV)


def check_digests(c, box, touched, before):
    """Pages of `touched` have their digests, the others are as they were."""
    want, got, old = pick.digests(c), box.double().cpu().numpy(), before.double().cpu().numpy()
    for page in range(c.pages):
        assert np.array_equal(got[page], want[page] if page in touched else old[page]), page


def pages_of(c, b, lo, hi):
    return {int(c.table[b, col]) for col in range(lo // c.page, -(-hi // c.page)) if hi > lo and 0 <= c.table[b, col] < c.pages}


@pytest.mark.parametrize("d,page", SIZES)
@pytest.mark.parametrize("form", ("f16", "bf16", "code4"))
def test_digests_of_prompts(form, d, page):
    """All tokens are new, and then only the last of them."""
    lens = [3 * page + 5, 1, 0, page, 2 * page - 1]
    c = ref.Cache(d + page, form, 2, d, page, lens, columns=5)
    t, codec = c.device()
    box = blank_digests(c)
    before = box.clone()
    print(f"digests {form} d={d} page={page}", flush=True)
    _pkg().kv_digest(t["pool"], box, t["table"], t["lengths"], starts=starts_of(lens), **codec)
    touched = set().union(*(pages_of(c, b, 0, n) for b, n in enumerate(lens)))
    check_digests(c, box, touched, before)
    _pkg().kv_digest(t["pool"], box, t["table"], t["lengths"], starts=starts_of(lens), **codec)      # once more: no change
    check_digests(c, box, touched, before)


@pytest.mark.parametrize("d,page", SIZES)
@pytest.mark.parametrize("form", ("f16", "bf16", "code4"))
@pytest.mark.parametrize("step", (1, 3, 40))
def test_digests_grow_with_the_rows(form, d, page, step):
    """Rows arrive a few at a time; after each arrival the digests are those of the tokens so far."""
    c = ref.Cache(d + step, form, 1, d, page, [70, 33, 0], columns=8)
    whole = list(c.lens)
    t, codec = c.device()
    box = blank_digests(c)
    lens = [70 - 42, 33 - 33, 0]
    c.lens = lens
    _pkg().kv_digest(t["pool"], box, t["table"], ints(lens), starts=starts_of(lens), **codec)
    while lens != whole:
        news = [min(step, w - n) for w, n in zip(whole, lens)]
        before = box.clone()
        lens = [n + m for n, m in zip(lens, news)]
        c.lens = lens
        if step == 1 and all(news[:2]):
            _pkg().kv_digest(t["pool"], box, t["table"][:2], ints(lens[:2]), **codec)
        else:
            _pkg().kv_digest(t["pool"], box, t["table"], ints(lens), starts=starts_of(news), **codec)
        check_digests(c, box, set().union(*(pages_of(c, b, n - m, n) for b, (n, m) in enumerate(zip(lens, news)))), before)


@pytest.mark.parametrize("form", ("bf16", "code4"))
def test_digests_leave_out_what_is_not_there(form):
    """Missing pages, rows that were refused, lengths past the table, starts that make no sense."""
    lens = [40, 40, 40, 200]
    c = ref.Cache(5, form, 2, 64, 16, [40, 40, 40, 48], columns=3)
    c.table[0, 1], c.table[2, 2] = -1, c.pages + 7
    c.lens = [40, 40, 40, 48]
    t, codec = c.device()
    box = blank_digests(c)
    before = box.clone()
    news = [40, 40, 40, 200]
    _pkg().kv_digest(t["pool"], box, t["table"], ints(lens), starts=starts_of(news), asked=ints([40, 3, 40, 1]), granted=ints([40, 0, 40, 1]), **codec)
    touched = pages_of(c, 0, 0, 40) | pages_of(c, 2, 0, 40) | pages_of(c, 3, 0, 48)
    check_digests(c, box, touched, before)
    box = before.clone()
    _pkg().kv_digest(t["pool"], box, t["table"], ints([-4, 0, 17, 33]), asked=ints([1, 1, 1, 1]), granted=ints([1, 1, 0, 1]), **codec)
    changed = (box != before).flatten(1).any(1).nonzero()[:, 0].tolist()
    assert changed == [int(c.table[3, 2])]
    box = before.clone()
    _pkg().kv_digest(t["pool"], box, t["table"], ints(c.lens), starts=ints([9, 4, 2, 2, -3]), **codec)
    assert torch.equal(box, before)


@pytest.mark.parametrize("form", ("f16", "bf16"))
def test_digests_of_no_numbers(form):
    c = ref.Cache(6, form, 1, 96, 16, [23, 16])
    k = c.rows16[0]
    p, q = int(c.table[0, 0]), int(c.table[1, 0])
    k[p, 0, 3, 5] = float("nan")
    k[p, 0, 4, 6], k[p, 0, 5, 7] = float("inf"), -float("inf")
    k[q, 0, :, 9] = float("nan")
    k[int(c.table[0, 1]), 0, 7:] = float("nan")              # behind the row's end
    t, codec = c.device()
    box = blank_digests(c)
    before = box.clone()
    _pkg().kv_digest(t["pool"], box, t["table"], t["lengths"], starts=starts_of([23, 16]))
    check_digests(c, box, {p, q, int(c.table[0, 1])}, before)


@pytest.mark.parametrize("d,page", SIZES[:5])
@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("news", ([1, 1, 1, 1], [37, 5, 0, 1], [3, 2, 9, 4]))
def test_scores(form, kind, d, page, news):
    heads, group = (2, 3) if d < 192 else (1, 5)
    lens = [260, 5, 0, 70]
    c = ref.Cache(d + len(news), form, heads, d, page, lens, columns=260 // page + 3)
    if page < 128:
        c.table[0, 1] = -1
    t, codec = c.device()
    g = torch.Generator().manual_seed(d)
    q = torch.randn(sum(news), heads * group, d, generator=g).to(ref.TYPES[kind])
    box = torch.randn(c.pages, heads, 2, d, generator=g).sort(dim=2).values.to(torch.float16 if form == "code4" else ref.TYPES[form])
    where = {} if max(news) == 1 else {"starts": starts_of(news), "max_new": max(news)}
    print(f"scores {form} d={d} page={page} news={news}", flush=True)
    got = _pkg().kv_score(q.to(DEV), box.to(DEV), t["pool"], t["table"], t["lengths"], **where, **codec).double().cpu().numpy()
    want, bound = pick.scores(c, q, box, news)
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    fine = np.isfinite(want)
    assert (np.abs(got[fine] - want[fine]) <= bound[fine]).all()


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("group", (1, 2, 4, 7, 8, 16, 33))
@pytest.mark.parametrize("most", (17, 1))
def test_scores_of_strided_queries(form, kind, group, most):
    """Queries side by side with keys and values, a table with a stride, scores in a given place that rows past max_new keep."""
    lens, news = [500, 300], [20, 3]
    c = ref.Cache(group, form, 2, 64, 32, lens, columns=16)
    t, codec = c.device()
    wide = torch.randn(23, 2 * group + 4, 64, generator=torch.Generator().manual_seed(group)).to(ref.TYPES[kind]).to(DEV)
    q = wide[:, 2: 2 + 2 * group]
    box = torch.randn(c.pages, 2, 2, 64).sort(dim=2).values.to(torch.float16 if form == "code4" else ref.TYPES[form]).to(DEV)
    table = torch.full((2, 40), 3, dtype=torch.int32, device=DEV)
    table[:, :16] = t["table"]
    out = torch.full((23, 2, 16), 5.0, device=DEV)
    _pkg().kv_score(q, box, t["pool"], table[:, :16], t["lengths"], starts=starts_of(news), max_new=most, out=out, **codec)
    want, bound = pick.scores(c, q, box, news)
    got = out.double().cpu().numpy()
    rows = [r for r in range(23) if r < most or 20 <= r < 20 + most]
    rest = [r for r in range(23) if r not in rows]
    assert (got[rest] == 5).all()
    fine = np.isfinite(want)
    fine[rest] = False
    assert np.array_equal(np.isneginf(got[rows]), np.isneginf(want[rows])) and (np.abs(got[fine] - want[fine]) <= bound[fine]).all()


@pytest.mark.parametrize("kind", ("f16", "bf16"))
@pytest.mark.parametrize("group", (1, 4, 16))
@pytest.mark.parametrize("d", (64, 96, 128, 192, 256))
def test_scores_over_codes_of_whole_groups(d, group, kind):
    """Every head size where sides come straight from the queries: large, small and zero rows, more rows than a workgroup's, an odd number of heads."""
    lens, news = [900, 77], [61, 14]
    c = ref.Cache(d, "code4", 3, d, 32, lens, columns=40)
    t, codec = c.device()
    g = torch.Generator().manual_seed(d + group)
    q = torch.randn(75, 3 * group, d, generator=g)
    q[3] *= 1000.0
    q[17, ::2] *= 2.0 ** -12
    q[18], q[19, 0] = 0.0, 0.0
    q = q.to(ref.TYPES[kind])
    box = torch.randn(c.pages, 3, 2, d, generator=g).sort(dim=2).values.to(torch.float16)
    got = _pkg().kv_score(q.to(DEV), box.to(DEV), t["pool"], t["table"], t["lengths"], starts=starts_of(news), max_new=61, **codec).double().cpu().numpy()
    want, bound = pick.scores(c, q, box, news)
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    fine = np.isfinite(want)
    assert (np.abs(got[fine] - want[fine]) <= bound[fine]).all()


@pytest.mark.parametrize("form", ("f16", "code4"))
def test_scores_bound_the_products(form):
    """What the scores are for: no key of the page has a larger product, summed over the group's heads."""
    lens = [200]
    c = ref.Cache(3, form, 1, 64, 16, lens)
    t, codec = c.device()
    box = blank_digests(c)
    _pkg().kv_digest(t["pool"], box, t["table"], t["lengths"], starts=starts_of(lens), **codec)
    q = torch.randn(1, 4, 64, generator=torch.Generator().manual_seed(2)).half()
    got = _pkg().kv_score(q.to(DEV), box, t["pool"], t["table"], t["lengths"], **codec)[0, 0].cpu().numpy()
    k = c.rows(0, 0, 0, 200)
    products = q[0].double().numpy() @ k.T
    for col in range(13):
        most = products[:, 16 * col: 16 * col + 16].max(1).sum()
        assert got[col] >= most - 2.0 ** -9 * np.abs(products).max() * 4


def run_select(scores, lens, news, page, count, first=1, last=1, **where):
    starts = None if all(m == 1 for m in news) and len(news) == scores.shape[0] else starts_of(news)
    return _pkg().kv_select(scores.to(DEV), ints(lens), page, count, starts=starts, first=first, last=last, **where).cpu().numpy()


@pytest.mark.parametrize("page,count", [(16, 1), (16, 7), (64, 32), (16, 200), (128, 4096), (1024, 3)])
@pytest.mark.parametrize("kind", ("random", "ties", "few values", "holes", "negative", "narrow"))
def test_select(page, count, kind):
    lens, news = [3000, 17, 0, 260, 1], [3, 17, 0, 2, 1]
    columns, rows = 300, 23
    g = torch.Generator().manual_seed(page + count)
    s = torch.randn(rows, 2, columns, generator=g)
    if kind == "ties":
        s = torch.zeros_like(s)
    elif kind == "few values":
        s = torch.randint(-2, 3, s.shape, generator=g) * 0.5 * torch.where(torch.rand(s.shape, generator=g) < 0.5, -1.0, 1.0)      # both zeros among them
    elif kind == "holes":
        s = torch.where(torch.rand(s.shape, generator=g) < 0.6, -torch.inf, s)
        s[torch.rand(s.shape, generator=g) < 0.1] = torch.nan
        s[torch.rand(s.shape, generator=g) < 0.05] = torch.inf
    elif kind == "negative":
        s = -1e30 * (1 + torch.rand(s.shape, generator=g))
    elif kind == "narrow":
        s = 1 + torch.randint(0, 40, s.shape, generator=g) * 2.0 ** -23
    for first, last in ((0, 0), (1, 1), (0, 1), (2, 1)):
        if first + last <= count:
            got = run_select(s, lens, news, page, count, first, last)
            assert np.array_equal(got, pick.select(s.numpy(), lens, news, page, count, first, last)), (first, last)


@pytest.mark.parametrize("columns", (1, 63, 64, 65, 1000, 2047, 4100, 9000))
@pytest.mark.parametrize("count", (2, 64, 1500))
def test_select_of_long_rows(columns, count):
    lens, news = [columns * 16, columns * 16 - 15, 16], [1, 1, 1]
    s = torch.randn(3, 3, columns, generator=torch.Generator().manual_seed(columns)).round(decimals=2)
    assert np.array_equal(run_select(s, lens, news, 16, count), pick.select(s.numpy(), lens, news, 16, count, 1, 1))


def test_select_rows_of_no_sequence():
    """Rows outside the starts, sequences with more rows than tokens, lengths past the columns, no sequence at all."""
    s = torch.randn(9, 2, 4)
    got = _pkg().kv_select(s.to(DEV), ints([2, 4000]), 16, 3, starts=ints([1, 5, 8])).cpu().numpy()
    want = np.full((9, 2, 3), -1, np.int32)
    want[3:5, :, 0] = 0                       # positions -2, -1, 0, 1: rows 1 .. 4
    want[5:8] = pick.select(s[5:8].numpy(), [64], [3], 16, 3, 1, 1)
    assert np.array_equal(got, want)
    out = torch.full((2, 2, 3), 9, dtype=torch.int32, device=DEV)
    assert _pkg().kv_select(s[:2].contiguous().to(DEV), ints([]), 16, 3, starts=ints([0]), out=out) is out
    assert (out == -1).all()
