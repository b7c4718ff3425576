"""Attention over chosen pages against float64, row by row: every format and head size, pages shared out over several workgroups and not, lists
with holes, repeats and pages behind the row, what is no number in places that nobody sees."""
import numpy as np
import pytest

import kv_pick_reference as pick
import kv_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FORMS = [("f16", "f16"), ("bf16", "bf16"), ("code4", "bf16"), ("code4", "f16")]


def _pkg():
    import paper_2605_17415_amd as pkg
    return pkg


def starts_of(news):
    return torch.tensor([0] + list(np.cumsum(news)), dtype=torch.int32, device=DEV)


def queries(seed, rows, heads, d, dtype):
    return (torch.randn(rows, heads, d, generator=torch.Generator().manual_seed(seed)) * 1.5).to(dtype).to(DEV)


def lists(c, rows, count, seed=0):
    """Ascending columns, some lists short; columns behind the row's position among them."""
    rng = np.random.default_rng(seed)
    out = np.full((rows, c.heads, count), -1, np.int32)
    for r in range(rows):
        for h in range(c.heads):
            n = int(rng.integers(0, min(count, c.columns) + 1)) if rng.random() < 0.3 else min(count, c.columns)
            out[r, h, :n] = np.sort(rng.permutation(c.columns)[:n])
    return out


def run(c, q, chosen, news=None, want_lse=True, **more):
    t, codec = c.device()
    lse = torch.full(q.shape[:2], 5.0, device=DEV) if want_lse else None
    where = {} if news is None else {"starts": starts_of(news), "max_new": max(news)}
    out = _pkg().kv_attend_pages(q, t["pool"], t["table"], t["lengths"], torch.from_numpy(chosen).to(DEV), lse=lse, **where, **more, **codec)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("d,page", [(64, 16), (96, 32), (128, 64), (128, 16), (192, 16), (256, 128)])
@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("count", (1, 2, 5, 30))
def test_one_token(form, kind, d, page, count):
    heads, group = (2, 3) if d < 192 else (1, 4)
    lens = [700, 20, 0, 1, 333]
    c = ref.Cache(d + count, form, heads, d, page, lens)
    q = queries(d, len(lens), heads * group, d, ref.TYPES[kind])
    chosen = lists(c, len(lens), count, d)
    print(f"one token {form} {kind} d={d} page={page} count={count}", flush=True)
    out, lse = run(c, q, chosen)
    pick.check_attention(c, q.cpu(), out, [1] * len(lens), chosen, lse)


@pytest.mark.parametrize("d,page", [(64, 16), (96, 16), (128, 64), (192, 32), (256, 16)])
@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("news", ([3, 5, 0, 4, 1], [150, 67, 41, 2, 1]))
def test_several_tokens(form, kind, d, page, news):
    """Prompts and chunks, sequences without new rows and with fewer tokens than rows."""
    lens = [260, 90, 40, 600, 0] if sum(news) < 20 else [150, 260, 40, 1, 0]
    c = ref.Cache(d, form, 2, d, page, lens)
    q = queries(d, sum(news), 4, d, ref.TYPES[kind])
    chosen = lists(c, sum(news), 6, d)
    print(f"several tokens {form} {kind} d={d} page={page}", flush=True)
    out, lse = run(c, q, chosen, news)
    pick.check_attention(c, q.cpu(), out, news, chosen, lse)


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("group", (1, 8, 16, 17, 64))
def test_heads_of_a_group(form, kind, group):
    c = ref.Cache(group, form, 2, 128, 32, [130, 700])
    q = queries(group, 2, 2 * group, 128, ref.TYPES[kind])
    chosen = lists(c, 2, 9, group)
    out, lse = run(c, q, chosen)
    pick.check_attention(c, q.cpu(), out, [1, 1], chosen, lse)


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("page", (16, 32, 1024))
def test_many_rows_without_shares(form, kind, page):
    """More (row, head) pairs than workgroups fit the chip: each is finished by one workgroup."""
    n = 500
    c = ref.Cache(n, form, 3, 64, page, [n], columns=-(-n // page) + 2)
    q = queries(n, n, 3, 64, ref.TYPES[kind])
    chosen = lists(c, n, 7, page)
    out, lse = run(c, q, chosen, [n])
    pick.check_attention(c, q.cpu(), out, [n], chosen, lse)


@pytest.mark.parametrize("form,kind", FORMS[:3])
def test_lists_of_any_content(form, kind):
    """Repeats, order that falls, numbers out of range, pages that the table does not have: each is passed over."""
    c = ref.Cache(1, form, 1, 64, 16, [300], columns=19)
    c.table[0, 5], c.table[0, 6] = -1, c.pages
    chosen = np.array([[[3, 3, 2, 7, 7, 5, 6, 8, -9, 4000, 1, 9, -1]], [[-5, 18, 18, 18, 2, 3, 1 << 30, -(1 << 31), 0, 0, 0, 0, 0]],
                       [[5, 6, 5, 6, 0, 1, 2, -1, -1, -1, -1, -1, -1]], [[0, 0, 0, 1, 2, 18, 17, 16, -1, -1, 2, 1, 0]]], np.int32)
    q = queries(1, 4, 2, 64, ref.TYPES[kind])
    out, lse = run(c, q, chosen, [4])
    pick.check_attention(c, q.cpu(), out, [4], chosen, lse)


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("new", (1, 20))
def test_every_page_chosen_is_attention_over_the_cache(form, kind, new):
    lens = [900, 33]
    c = ref.Cache(new, form, 2, 128, 16, lens)
    news = [new, new]
    q = queries(new, 2 * new, 8, 128, ref.TYPES[kind])
    chosen = np.broadcast_to(np.arange(c.columns, dtype=np.int32), (2 * new, 2, c.columns)).copy()
    out, lse = run(c, q, chosen, news)
    pick.check_attention(c, q.cpu(), out, news, chosen, lse)
    ref.check_attention(c, q.cpu(), out, news, lse=lse)


@pytest.mark.parametrize("form,kind", FORMS[:3])
def test_no_numbers_where_nobody_looks(form, kind):
    """Pages that are not chosen, tokens behind the row, pages of other sequences: anything may stand there."""
    lens, news = [150, 90], [3, 2]
    c = ref.Cache(9, form, 1, 64, 16, lens, spare=4)
    q = queries(9, 5, 2, 64, ref.TYPES[kind])
    chosen = np.full((5, 1, 6), -1, np.int32)
    chosen[:, 0, :4] = [0, 4, 5, 9]
    chosen[3:, 0, :3], chosen[3:, 0, 3] = [1, 3, 5], -1
    want, _ = run(c, q, chosen, news)
    t, codec = c.device()
    pool = t["pool"]
    used = {int(c.table[0, x]) for x in (0, 4, 5, 9)} | {int(c.table[1, x]) for x in (1, 3, 5)}
    bad = torch.tensor([p not in used for p in range(c.pages)], device=DEV)
    if form == "code4":
        pool[bad] = 255                                     # norms that are no numbers
        half = 16 * 64
        last = pool[int(c.table[0, 9])]
        norms = last[:, half:].view(torch.float16)
        norms[:, 6:16], norms[:, 22:] = torch.nan, torch.inf
    else:
        pool[bad] = torch.nan
        last = pool[int(c.table[0, 9])]
        last[:, 0, 6:] = torch.nan
        last[:, 1].view(1, 2, 64, 8)[:, 0, :, 6:] = torch.inf
        last[:, 1].view(1, 2, 64, 8)[:, 1] = torch.nan
    got = _pkg().kv_attend_pages(q, pool, t["table"], t["lengths"], torch.from_numpy(chosen).to(DEV), starts=starts_of(news), max_new=3, **codec)
    assert torch.equal(got, want)


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("page", (16, 32))
def test_no_numbers_in_a_neighbours_page(form, kind, page):
    """Neighbouring rows are worked on together: what one of them has chosen may be anything to the others."""
    n, new = 9 * page, 8
    c = ref.Cache(7, form, 1, 64, page, [n], spare=2)
    q = queries(7, new, 2, 64, ref.TYPES[kind])
    chosen = np.full((new, 1, 5), -1, np.int32)
    for r in range(new):
        chosen[r, 0, :4] = [0, 2 + r % 3, 5, 8]
    chosen[3, 0] = [0, 1, 2, 7, 8]                          # page 1 and page 7 are row 3's alone, page 6 is nobody's
    want, _ = run(c, q, chosen, [new])
    t, codec = c.device()
    for col in (1, 6, 7):
        p = int(c.table[0, col])
        t["pool"][p] = 255 if form == "code4" else torch.nan
    got = _pkg().kv_attend_pages(q, t["pool"], t["table"], t["lengths"], torch.from_numpy(chosen).to(DEV), starts=starts_of([new]), max_new=new, **codec)
    others = [r for r in range(new) if r != 3]
    assert torch.equal(got[others], want[others]) and not torch.isfinite(got[3].float()).all()
    if form != "code4":                                     # infinite values, that only row 3 sees
        clean, _ = c.device()
        p = int(c.table[0, 7])
        clean["pool"][p, 0, 1] = torch.inf
        got = _pkg().kv_attend_pages(q, clean["pool"], t["table"], t["lengths"], torch.from_numpy(chosen).to(DEV), starts=starts_of([new]), max_new=new, **codec)
        assert torch.equal(got[others], want[others]) and torch.isinf(got[3].float()).all()


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("group", (1, 2, 5, 9))
def test_neighbours_that_choose_alike_and_not(form, kind, group):
    """Units of 16, 8, 3 and 1 rows; sequences that begin and end inside one, more rows than tokens, columns past a word of bits."""
    lens, news = [1300, 40, 700, 5], [37, 1, 20, 9]
    c = ref.Cache(group, form, 2, 64, 16, lens, columns=90)
    rows = sum(news)
    q = queries(group, rows, 2 * group, 64, ref.TYPES[kind])
    rng = np.random.default_rng(group)
    chosen = np.full((rows, 2, 9), -1, np.int32)
    for r in range(rows):
        for h in range(2):
            own = {0, int(rng.integers(0, 80)), int(rng.integers(0, 80)), 3 + (r + h) // 4, 40 + r % 3, 79}
            chosen[r, h, : len(own)] = sorted(own)
    out, lse = run(c, q, chosen, news)
    pick.check_attention(c, q.cpu(), out, news, chosen, lse)


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("scale", (0.0, -0.3, 2.0))
def test_scale(form, kind, scale):
    c = ref.Cache(4, form, 1, 64, 16, [200, 77])
    q = queries(4, 2, 2, 64, ref.TYPES[kind])
    chosen = lists(c, 2, 5, 4)
    out, _ = run(c, q, chosen, scale=scale, want_lse=False)
    pick.check_attention(c, q.cpu(), out, [1, 1], chosen, scale=scale)


@pytest.mark.parametrize("form,kind", FORMS[:3])
def test_strides_and_rows_that_keep_what_they_have(form, kind):
    """Queries and results inside wider rows, rows of no sequence and past max_new."""
    lens, news = [200, 90], [6, 2]
    c = ref.Cache(8, form, 2, 64, 32, lens)
    wide = queries(8, 11, 10, 64, ref.TYPES[kind])
    q = wide[:, 3:7]
    place = torch.full((11, 9, 64), 3.0, dtype=q.dtype, device=DEV)
    t, codec = c.device()
    chosen = lists(c, 11, 4, 8)
    starts = torch.tensor([1, 7, 9], dtype=torch.int32, device=DEV)
    _pkg().kv_attend_pages(q, t["pool"], t["table"], t["lengths"], torch.from_numpy(chosen).to(DEV), starts=starts, max_new=4, out=place[:, 2:6], **codec)
    assert (place[:, :2] == 3).all() and (place[:, 6:] == 3).all()
    assert (place[[0, 5, 6, 9, 10]] == 3).all()
    rows = [1, 2, 3, 4, 7, 8]
    full = torch.zeros(8, 4, 64, dtype=q.dtype)
    full[[0, 1, 2, 3, 6, 7]] = place[rows, 2:6].cpu()
    want = chosen[1:9].copy()
    want[4:6] = -1                                           # rows without a result: compared as rows that see nothing
    pick.check_attention(c, q[1:9].cpu(), full, news, want)


@pytest.mark.parametrize("form,kind", FORMS[:3])
def test_equal_calls_give_equal_bits(form, kind):
    c = ref.Cache(2, form, 2, 128, 64, [3000, 1500])
    q = queries(2, 2, 8, 128, ref.TYPES[kind])
    chosen = lists(c, 2, 20, 2)
    a, la = run(c, q, chosen)
    b, lb = run(c, q, chosen)
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_pool_past_four_gigabytes():
    """Page numbers whose bytes lie past 2^32."""
    pages, heads, d, page = 2200, 8, 128, 512
    pool = torch.zeros(pages, heads, 2, page, d, dtype=torch.bfloat16, device=DEV)
    for p in (0, pages - 1):
        pool[p] = torch.randn(heads, 2, page, d, device=DEV).bfloat16()
    table = torch.tensor([[pages - 1, 5, pages - 1], [0, 5, 0]], dtype=torch.int32, device=DEV)
    lengths = torch.tensor([3 * page, 3 * page], dtype=torch.int32, device=DEV)
    low = pool[[0, pages - 1]].contiguous()
    small = torch.tensor([[1, -1, 1], [0, -1, 0]], dtype=torch.int32, device=DEV)
    q = torch.randn(2, 16, d, device=DEV).bfloat16()
    chosen = torch.tensor([0, 2], dtype=torch.int32, device=DEV).expand(2, heads, 2).contiguous()
    a = _pkg().kv_attend_pages(q, pool, table, lengths, chosen)
    b = _pkg().kv_attend_pages(q, low, small, lengths, chosen)
    assert torch.equal(a, b)
    box, few = torch.zeros(pages, heads, 2, d, dtype=torch.bfloat16, device=DEV), torch.zeros(2, heads, 2, d, dtype=torch.bfloat16, device=DEV)
    starts = torch.tensor([0, 3 * page, 6 * page], dtype=torch.int32, device=DEV)
    _pkg().kv_digest(pool, box, table, lengths, starts=starts)
    _pkg().kv_digest(low, few, small, lengths, starts=starts)
    assert torch.equal(box[[0, pages - 1]], few) and bool((few != 0).any())
