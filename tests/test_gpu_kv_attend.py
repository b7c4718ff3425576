"""Attention over the paged cache against float64, row by row: both kernels (few and many new rows), every format and head size, lengths
from nothing to several shares, windows, first tokens, missing pages, what is no number in places that nobody sees."""
import math

import numpy as np
import pytest

import kv_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _pkg():
    import paper_2605_17415_amd as pkg
    return pkg


def starts_of(news):
    return torch.tensor([0] + list(np.cumsum(news)), dtype=torch.int32, device=DEV)


def queries(seed, rows, heads, d, dtype):
    return (torch.randn(rows, heads, d, generator=torch.Generator().manual_seed(seed)) * 1.5).to(dtype).to(DEV)


def run(c, q, news=None, want_lse=True, **mask):
    t, codec = c.device()
    lse = torch.full(q.shape[:2], 5.0, device=DEV) if want_lse else None
    where = {} if news is None else {"starts": starts_of(news), "max_new": max(news)}
    out = _pkg().kv_attend(q, t["pool"], t["table"], t["lengths"], lse=lse, **where, **mask, **codec)
    torch.cuda.synchronize()
    return out, lse


FORMS = [("f16", "f16"), ("bf16", "bf16"), ("code4", "bf16"), ("code4", "f16")]


@pytest.mark.parametrize("d,page", [(64, 16), (96, 32), (128, 64), (192, 16), (256, 128)])
@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("lens", ([1], [0, 33, 7], [513, 16, 1200, 0, 1]))
def test_one_token(form, kind, d, page, lens):
    heads, group = (2, 3) if d < 192 else (1, 4)
    c = ref.Cache(d + len(lens), form, heads, d, page, lens)
    q = queries(d, len(lens), heads * group, d, ref.TYPES[kind])
    print(f"one token {form} d={d} page={page} lens={lens}", flush=True)
    out, lse = run(c, q)
    ref.check_attention(c, q.cpu(), out, [1] * len(lens), lse=lse)


@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 3), (64, 4), (100, 40), (31, 600), (5000, 2)])
def test_one_token_with_a_window(form, kind, window, sinks):
    lens = [700, 20, 65, 0, 300]
    c = ref.Cache(window, form, 2, 64, 16, lens)
    q = queries(window, len(lens), 4, 64, ref.TYPES[kind])
    out, lse = run(c, q, window=window, sinks=sinks)
    ref.check_attention(c, q.cpu(), out, [1] * len(lens), lse=lse, window=window, sinks=sinks)


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("group", (1, 8, 16, 17, 64))
def test_heads_of_a_group(form, kind, group):
    c = ref.Cache(group, form, 2, 128, 32, [130, 700])
    q = queries(group, 2, 2 * group, 128, ref.TYPES[kind])
    out, lse = run(c, q)
    ref.check_attention(c, q.cpu(), out, [1, 1], lse=lse)


@pytest.mark.parametrize("d,page", [(64, 16), (96, 16), (128, 64), (192, 32), (256, 16)])
@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 5)])
def test_several_tokens(form, kind, d, page, window, sinks):
    """Few rows: a handful of new tokens a sequence, among them sequences without any and with fewer tokens than rows."""
    lens, news = [90, 3, 40, 600, 0], [3, 5, 0, 4, 1]
    c = ref.Cache(d, form, 2, d, page, lens)
    q = queries(d, sum(news), 4, d, ref.TYPES[kind])
    out, lse = run(c, q, news, window=window, sinks=sinks)
    ref.check_attention(c, q.cpu(), out, news, lse=lse, window=window, sinks=sinks)


@pytest.mark.parametrize("d,page", [(64, 16), (96, 16), (128, 64), (192, 32), (256, 16)])
@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 5), (1, 0), (70, 130)])
def test_many_tokens(form, kind, d, page, window, sinks):
    lens, news = [150, 260, 40, 0, 1], [150, 67, 41, 2, 1]
    c = ref.Cache(d + window, form, 1, d, page, lens)
    q = queries(d, sum(news), 3, d, ref.TYPES[kind])
    print(f"many tokens {form} d={d} page={page} window={window}", flush=True)
    out, lse = run(c, q, news, window=window, sinks=sinks)
    ref.check_attention(c, q.cpu(), out, news, lse=lse, window=window, sinks=sinks)


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("new", (1, 65))
def test_missing_pages(form, kind, new):
    """Entries that name no page hold no visible token; a sequence without any page sees nothing."""
    lens, news = [200, 150, 100], [new, new, new]
    c = ref.Cache(1, form, 2, 64, 16, lens)
    c.table[0, 2], c.table[0, 5], c.table[1, 0] = -1, c.pages, -2 ** 31
    c.table[2] = -1
    q = queries(1, 3 * new, 4, 64, ref.TYPES[kind])
    out, lse = run(c, q, news)
    ref.check_attention(c, q.cpu(), out, news, lse=lse)
    assert (out[2 * new:] == 0).all()


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("new,window,sinks", [(1, 0, 0), (1, 40, 3), (70, 0, 0), (70, 40, 3), (3, 0, 0), (3, 40, 3)])
def test_no_numbers_where_nobody_looks(form, kind, new, window, sinks):
    """Everything that no row of a sequence sees is NaN or infinite: the pages' ends, what lies before the window, free pages."""
    lens = [133, 81]
    c = ref.Cache(2, form, 2, 64, 16, lens)
    q = queries(2, 2 * new, 4, 64, ref.TYPES[kind])
    hidden = np.ones((c.pages, c.page), bool)
    for b, n in enumerate(lens):
        for t in range(n):
            if not window or t > n - new - window or t < sinks:
                hidden[c.table[b, t // c.page], t % c.page] = False
    for p, t in zip(*np.nonzero(hidden)):
        bad = (float("nan"), float("inf"), float("-inf"))[(p + t) % 3]
        if form == "code4":
            c.norms[:, p, :, t] = bad
        else:
            c.rows16[:, p, :, t] = bad
    out, lse = run(c, q, [new, new], window=window, sinks=sinks)
    shown = ref.Cache(2, form, 2, 64, 16, lens)
    ref.check_attention(shown, q.cpu(), out, [new, new], lse=lse, window=window, sinks=sinks)


@pytest.mark.parametrize("form", ("f16", "bf16", "code4"))
@pytest.mark.parametrize("bad", (float("nan"), float("inf")))
@pytest.mark.parametrize("new", (6, 100))
def test_no_number_in_a_later_token_leaves_earlier_rows_alone(form, bad, new):
    """A token that only the later rows see: rows before it have the results that they have without it."""
    c = ref.Cache(3, form, 1, 64, 16, [new + 40])
    q = queries(3, new, 2, 64, ref.TYPES["bf16" if form == "code4" else form])
    want, _ = run(c, q, [new])
    at = new + 40 - 3                                       # seen by the last three rows
    if form == "code4":
        c.norms[:, c.table[0, at // 16], :, at % 16] = bad
    else:
        c.rows16[:, c.table[0, at // 16], :, at % 16, 5] = bad
    got, _ = run(c, q, [new])
    assert torch.equal(got[:-3], want[:-3])
    assert not torch.isfinite(got[-3:]).all()


@pytest.mark.parametrize("form,kind", FORMS[:3])
def test_long_sequences_in_many_shares(form, kind):
    """Long enough that a pair is split over many workgroups, next to short ones; large scores at either end of the cache."""
    lens = [20_011, 5, 4096, 777]
    c = ref.Cache(4, form, 1, 64, 64, lens)
    if form != "code4":
        c.rows16[0, c.table[0, 0], 0, 3] *= 4
        c.rows16[0, c.table[0, -1], 0, 1] *= 4
    q = queries(4, 4, 4, 64, ref.TYPES[kind])
    out, lse = run(c, q)
    ref.check_attention(c, q.cpu(), out, [1] * 4, lse=lse)
    again, _ = run(c, q)
    assert torch.equal(out, again)                          # no order of atomics in it


@pytest.mark.parametrize("d,page", [(64, 16), (96, 32), (128, 64), (256, 16)])
@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (900, 5)])
def test_a_chunk_after_a_long_beginning(form, kind, d, page, window, sinks):
    """Many new rows whose keys are shared out over several workgroups, next to a sequence without any and to a short one."""
    lens, news = [2300, 70, 9, 1500], [70, 66, 0, 40]
    c = ref.Cache(d, form, 1, d, page, lens)
    q = queries(d, sum(news), 2, d, ref.TYPES[kind])
    out, lse = run(c, q, news, window=window, sinks=sinks)
    ref.check_attention(c, q.cpu(), out, news, lse=lse, window=window, sinks=sinks)


@pytest.mark.parametrize("d,page", [(64, 16), (96, 64), (128, 128), (192, 32), (256, 64)])
@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (2199, 4)])
def test_both_kernels_agree(form, kind, d, page, window, sinks):
    """The last rows of long chunks, as rows of the chunk and as few rows: the same operands, so only the weights' rounding (2^-11, 2^-8;
    a few 2^-24 for each token's score and sum) and the result's own may differ.  Many workgroups and many tiles, several times."""
    pkg = _pkg()
    heads, group, lens, news = 4, 4, [5000, 3100, 900], [500, 756, 300]
    c = ref.Cache(17, form, heads, d, page, lens)
    t, codec = c.device()
    q = queries(17, sum(news), heads * group, d, ref.TYPES[kind])
    last = 3
    rows = torch.cat([torch.arange(e - last, e) for e in np.cumsum(news)]).to(DEV)
    few = pkg.kv_attend(q[rows], t["pool"], t["table"], t["lengths"], starts=starts_of([last] * 3), max_new=last, window=window, sinks=sinks, **codec)
    for _ in range(3):
        many = pkg.kv_attend(q, t["pool"], t["table"], t["lengths"], starts=starts_of(news), max_new=max(news), window=window, sinks=sinks, **codec)
        torch.cuda.synchronize()
        far = (many[rows].double() - few.double()).norm(dim=-1)
        # the values are independent rows, so the result's length is about |w|_2 |v|, and roundings of at most `step` of each weight, independent
        # in the two kernels, move it by at most that times sqrt(2) step in the mean square: five times step leaves three standard
        # deviations and a result a third shorter than the mean
        step = 2.0 ** -11 if form == "code4" else ref.HALF[few.dtype]
        size = few.double().norm(dim=-1)
        assert (far <= (2 * ref.HALF[few.dtype] + 5 * step) * size + 2.0 ** -18 * math.sqrt(d)).all(), float((far / size).max())


@pytest.mark.parametrize("form,kind", FORMS[:3])
@pytest.mark.parametrize("lens", ([40, 0, 5], [1800, 700]))
def test_more_heads_than_few_rows(form, kind, lens):
    """One token of a group of 72 heads: the kernel of many rows, without starts."""
    c = ref.Cache(14, form, 1, 64, 16, lens)
    q = queries(14, len(lens), 72, 64, ref.TYPES[kind])
    out, lse = run(c, q)
    ref.check_attention(c, q.cpu(), out, [1] * len(lens), lse=lse)


@pytest.mark.parametrize("form", ("bf16", "code4"))
def test_rows_without_a_result(form):
    """Rows past max_new and rows of no sequence get none; the others' results do not change."""
    lens, news = [1200, 90], [100, 90]
    c = ref.Cache(15, form, 1, 64, 16, lens)
    q = queries(15, sum(news) + 6, 2, 64, torch.bfloat16)
    t, codec = c.device()
    starts = starts_of(news) + 3                            # rows 0 .. 2 and the last three belong to nobody
    want = _pkg().kv_attend(q, t["pool"], t["table"], t["lengths"], starts=starts, max_new=100, **codec)
    ref.check_attention(c, q[3:-3].cpu(), want[3:-3], news)
    out = torch.full_like(q, 3.0)
    _pkg().kv_attend(q, t["pool"], t["table"], t["lengths"], starts=starts, max_new=95, out=out, **codec)
    torch.cuda.synchronize()
    assert torch.equal(out[3:98], want[3:98]) and torch.equal(out[103:-3], want[103:-3])
    assert (out[:3] == 3).all() and (out[98:103] == 3).all() and (out[-3:] == 3).all()


def test_many_sequences():
    """More sequences than lanes: shares are found by scans over them."""
    lens = [int(x) for x in np.random.default_rng(0).integers(0, 200, 150)] + [900]
    c = ref.Cache(5, "bf16", 2, 64, 16, lens)
    q = queries(5, len(lens), 2, 64, torch.bfloat16)
    out, lse = run(c, q)
    ref.check_attention(c, q.cpu(), out, [1] * len(lens), lse=lse)


def test_far_offsets():
    """A pool past 2^32 bytes, pages at its end."""
    pkg = _pkg()
    heads, d, page = 4, 128, 64
    each = pkg.kv_page_bytes(1, page, heads, d)
    pages = (5 << 30) // each
    pool = torch.empty(pages, heads, 2, page, d, dtype=torch.bfloat16, device=DEV)
    pool[-40:].normal_()
    c = ref.Cache(6, "bf16", heads, d, page, [40 * page - 7], spare=0)
    c.rows16 = torch.zeros(2, 40, heads, page, d, dtype=torch.bfloat16)
    far = pool[-40:].cpu()
    c.pages = 40
    c.take(far)
    q = queries(6, 1, 8, d, torch.bfloat16)
    table = torch.from_numpy(c.table).to(DEV) + (pages - 40)
    out = pkg.kv_attend(q, pool, table, torch.tensor(c.lens, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    ref.check_attention(c, q.cpu(), out, [1])


@pytest.mark.parametrize("form", ("bf16", "code4"))
@pytest.mark.parametrize("new", (1, 80))
def test_strides_scale_and_an_own_output(form, new):
    pkg = _pkg()
    lens = [130, 90]
    c = ref.Cache(8, form, 2, 64, 32, lens)
    t, codec = c.device()
    qkv = torch.randn(2 * new, 12, 64, device=DEV).bfloat16()
    q = qkv[:, 4:8]                                         # heads inside a wider matrix
    out = torch.full((2 * new, 6, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    got = pkg.kv_attend(q, t["pool"], t["table"], t["lengths"], starts=starts_of([new, new]), max_new=new, scale=0.3, out=out[:, 1:5], **codec)
    torch.cuda.synchronize()
    assert got.data_ptr() == out[:, 1:5].data_ptr() and (out[:, 0] == 9).all() and (out[:, 5] == 9).all()
    ref.check_attention(c, q.cpu(), got, [new, new], scale=0.3)


@pytest.mark.parametrize("form", ("f16", "code4"))
def test_in_a_graph_and_on_another_stream(form):
    """Captured once, replayed with other lengths, tables and queries in the same tensors; eager work between the replays."""
    pkg = _pkg()
    c = ref.Cache(10, form, 2, 64, 16, [300, 80])
    t, codec = c.device()
    kind = ref.TYPES["f16"]
    q, k, v = queries(1, 2, 4, 64, kind), queries(2, 2, 2, 64, kind), queries(3, 2, 2, 64, kind)
    out = torch.empty_like(q)

    def step(pool):
        pkg.kv_append(pool, k, v, t["table"], t["lengths"], **codec)
        pkg.kv_attend(q, pool, t["table"], t["lengths"], out=out, **codec)

    step(t["pool"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            step(t["pool"])
    torch.cuda.current_stream().wait_stream(s)
    for n, lens in enumerate(([300, 80], [17, 1], [299, 64])):
        t["lengths"].copy_(torch.tensor(lens, dtype=torch.int32))
        q.copy_(queries(20 + n, 2, 4, 64, kind))
        k.copy_(queries(30 + n, 2, 2, 64, kind))
        torch.cuda.synchronize()
        other = t["pool"].clone()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step(other)
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(other, t["pool"])


def test_refusals_with_tensors():
    pkg = _pkg()
    c = ref.Cache(11, "bf16", 2, 64, 16, [20])
    t, _ = c.device()
    q = queries(1, 1, 4, 64, torch.bfloat16)
    good = (q, t["pool"], t["table"], t["lengths"])
    pkg.kv_attend(*good)
    for bad in ((q.half(), *good[1:]), (q[..., :32].contiguous(), *good[1:]), (q.float(), *good[1:]), (q[:, :3].contiguous(), *good[1:]),
                (torch.cat([q, q]), *good[1:]), (q, t["pool"][:, :, :1], *good[2:]), (q, t["pool"].transpose(0, 1), *good[2:]),
                (q, t["pool"], t["table"].long(), t["lengths"]), (q, t["pool"], t["table"], t["lengths"].repeat(2)), (q.cpu(), *good[1:]),
                (torch.empty(1, 4, 128, dtype=q.dtype, device=DEV)[..., ::2], *good[1:])):
        with pytest.raises((TypeError, ValueError, pkg.IvftqError)):
            pkg.kv_attend(*bad)
    with pytest.raises(pkg.IvftqError):
        pkg.kv_attend(*good, window=-1)
    with pytest.raises(ValueError):
        pkg.kv_attend(*good, out=torch.empty(1, 2, 64, dtype=q.dtype, device=DEV))
    with pytest.raises(ValueError):
        pkg.kv_attend(*good, lse=torch.empty(4, device=DEV))
    with pytest.raises((TypeError, ValueError)):
        pkg.kv_attend(*good, starts=torch.zeros(3, dtype=torch.int32, device=DEV))
    code = ref.Cache(11, "code4", 2, 64, 16, [20])
    t2, codec = code.device()
    for change in (dict(rotation=codec["rotation"][:32]), dict(rotation=codec["rotation"].double()), dict(levels=codec["levels"][:8]), dict(levels=codec["levels"] + 1)):
        with pytest.raises((ValueError, pkg.IvftqError)):
            pkg.kv_attend(q, t2["pool"], t2["table"], t2["lengths"], **{**codec, **change})


@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("new", (1, 70))
def test_a_heavy_token_without_a_value(form, kind, new):
    """A first token that takes all of the weight but a millionth and has next to no value: the result is made of the others.  Their
    roundings (a score's operands, the weight, for codes the value's levels: a few times `step` of each token's part) are independent, so
    they add up as squares: eight steps of the parts' root of squares, and the result's own rounding."""
    d, n = 64, 2000
    rng = np.random.default_rng(new)
    u = rng.standard_normal(d)
    u /= np.linalg.norm(u)
    c = ref.Cache(21, form, 1, d, 64, [n])
    p0 = c.table[0, 0]
    if form == "code4":
        z = c.rotation.astype(np.float64) @ u
        c.codes[0, p0, 0, 0] = np.abs(z[:, None] - c.levels[None].astype(np.float64)).argmin(1)
        c.norms[0] = math.sqrt(d)
        c.norms[0, p0, 0, 0], c.norms[1, p0, 0, 0] = 15.0, 2.0 ** -12
    else:
        c.rows16[0, p0, 0, 0] = torch.from_numpy(15 * u).to(c.rows16.dtype)
        c.rows16[1] *= 64
        c.rows16[1, p0, 0, 0] = 2.0 ** -12
    q = torch.from_numpy(8 * u + 0.3 * rng.standard_normal((new, 2, d))).to(ref.TYPES[kind]).to(DEV)
    got, _ = run(c, q, [new])
    k, v = c.rows(0, 0, 0, n), c.rows(1, 0, 0, n)
    size, step, out_step = np.linalg.norm(v, axis=1), 2.0 ** -11 if form == "code4" else ref.HALF[ref.TYPES[kind]], ref.HALF[ref.TYPES[kind]]
    for i in range(new):
        seen = n - new + i + 1
        for h in range(2):
            s = k[:seen] @ q[i, h].double().cpu().numpy() / math.sqrt(d)
            w = np.exp(s - s.max())
            assert s.argmax() == 0 and np.sort(w)[-2] < 0.01
            w /= w.sum()
            exact = w @ v[:seen]
            far = np.linalg.norm(got[i, h].double().cpu().numpy() - exact)
            may = 8 * step * math.sqrt(((w * size[:seen]) ** 2).sum()) + out_step * np.linalg.norm(exact) + 2.0 ** -25 * math.sqrt(d)
            assert far <= may, (i, h, far / may)


@pytest.mark.parametrize("kind", ("f16", "bf16"))
@pytest.mark.parametrize("new", (1, 70))
@pytest.mark.parametrize("power", (-12, 7))
def test_norms_of_any_size(kind, new, power):
    """Values' norms far from one, and from each other: float16 weights take no harm."""
    c = ref.Cache(22, "code4", 2, 64, 16, [900, 130])
    c.norms[1] = (c.norms[1].astype(np.float64) * 2.0 ** power * np.where(c.rng.random(c.norms[1].shape) < 0.1, 2.0 ** 4, 1)).astype(np.float16)
    q = queries(22, 2 * new, 4, 64, ref.TYPES[kind])
    if kind == "f16" and power < 0:
        kind = "bf16"                                       # such results are under what float16 holds well
        q = q.bfloat16()
    out, lse = run(c, q, [new, new])
    ref.check_attention(c, q.cpu(), out, [new, new], lse=lse)


@pytest.mark.parametrize("form,kind", FORMS[1:])
def test_more_row_tiles_than_lanes_share_the_workgroups(form, kind):
    """Shares are found by scans over all row tiles, 96 here, among them rows that see nothing and a sequence without rows."""
    lens, news = [3000, 100, 0, 1500], [3000, 100, 3, 700]
    c = ref.Cache(23, form, 1, 64, 64, lens)
    q = queries(23, sum(news), 1, 64, ref.TYPES[kind])
    out, lse = run(c, q, news)
    ref.check_attention(c, q.cpu(), out, news, lse=lse)
    again, _ = run(c, q, news)
    assert torch.equal(out, again)


def test_without_starts_one_row_a_sequence_whatever_max_new_says():
    c = ref.Cache(24, "bf16", 1, 64, 16, [900, 30])
    t, _ = c.device()
    q = queries(24, 2, 4, 64, torch.bfloat16)
    out = _pkg().kv_attend(q, t["pool"], t["table"], t["lengths"], max_new=500)
    torch.cuda.synchronize()
    ref.check_attention(c, q.cpu(), out, [1, 1])


@pytest.mark.parametrize("form,kind", FORMS[1:])
def test_a_chunk_in_a_graph(form, kind):
    """Rows written and attended over many keys, captured once and replayed with other lengths and rows; eager work between the replays."""
    pkg = _pkg()
    news = [90, 40]
    c = ref.Cache(25, form, 2, 64, 16, [1600, 900])
    t, codec = c.device()
    dtype = ref.TYPES[kind]
    q, k, v = queries(1, sum(news), 4, 64, dtype), queries(2, sum(news), 2, 64, dtype), queries(3, sum(news), 2, 64, dtype)
    out, lse, starts = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV), starts_of(news)

    def step(pool):
        pkg.kv_append(pool, k, v, t["table"], t["lengths"], starts=starts, **codec)
        pkg.kv_attend(q, pool, t["table"], t["lengths"], starts=starts, max_new=90, window=700, sinks=3, out=out, lse=lse, **codec)

    step(t["pool"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(t["pool"])
    for n, lens in enumerate(([1600, 900], [95, 40], [1111, 899])):
        t["lengths"].copy_(torch.tensor(lens, dtype=torch.int32))
        for x, seed in ((q, 40), (k, 50), (v, 60)):
            x.copy_(queries(seed + n, x.shape[0], x.shape[1], 64, dtype))
        torch.cuda.synchronize()
        other = t["pool"].clone()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        step(other)
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], lse) and torch.equal(other, t["pool"])


@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("d", (64, 128))
def test_row_tiles_in_shares_agree_with_few_rows(form, kind, d):
    """Enough keys a head that its row tiles are dealt out in shares of more than 64 tiles, most of them cut: the last rows against the
    kernel of few rows, as in test_both_kernels_agree."""
    pkg = _pkg()
    heads, group, page, lens, news = 32, 4, 64, [20_000, 3000], [100, 40]
    need = [-(-n // page) for n in lens]
    g = torch.Generator(device=DEV).manual_seed(d)
    table = torch.full((2, max(need)), -1, dtype=torch.int32, device=DEV)
    order = torch.randperm(sum(need), generator=g, device=DEV).int()
    table[0], table[1, :need[1]] = order[:need[0]], order[need[0]:]
    codec = {}
    if form == "code4":
        pool = torch.randint(0, 256, (sum(need), heads, page * (d + 4)), generator=g, device=DEV, dtype=torch.uint8)
        norms = ((torch.rand(sum(need), heads, 2 * page, generator=g, device=DEV) + 0.5) * math.sqrt(d)).half()
        pool[..., page * d:] = norms.view(torch.uint8)
        codec = {"rotation": torch.from_numpy(pkg.ivftq_haar_rotation(d, 3)).to(DEV), "levels": pkg.ivftq_build_codebook(4, d)[0]}
    else:
        pool = torch.randn(sum(need), heads, 2, page, d, generator=g, device=DEV).to(ref.TYPES[form])
    lengths = torch.tensor(lens, dtype=torch.int32, device=DEV)
    q = queries(d, sum(news), heads * group, d, ref.TYPES[kind])
    last = 3
    rows = torch.cat([torch.arange(e - last, e) for e in np.cumsum(news)]).to(DEV)
    logs, few_logs = torch.empty(q.shape[:2], device=DEV), torch.empty(2 * last, heads * group, device=DEV)
    few = pkg.kv_attend(q[rows], pool, table, lengths, starts=starts_of([last] * 2), max_new=last, lse=few_logs, **codec)
    many = pkg.kv_attend(q, pool, table, lengths, starts=starts_of(news), max_new=max(news), lse=logs, **codec)
    torch.cuda.synchronize()
    far, size = (many[rows].double() - few.double()).norm(dim=-1), few.double().norm(dim=-1)
    step = 2.0 ** -11 if form == "code4" else ref.HALF[few.dtype]
    assert (far <= (2 * ref.HALF[few.dtype] + 5 * step) * size + 2.0 ** -18 * math.sqrt(d)).all(), float((far / size).max())
    assert (logs[rows] - few_logs).abs().max() <= 1e-4
