"""Scores of pages whose digests are not all finite numbers: one rule for one new row and for several, so that a decoding step and a chunk over
the same cache choose the same pages."""
import numpy as np
import pytest

import kv_pick_reference as pick
import kv_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FORMS = [("f16", "f16"), ("bf16", "bf16"), ("code4", "bf16"), ("code4", "f16")]
PAGE, COLUMNS = 16, 12
INF = np.inf


def _pkg():
    import paper_2605_17415_amd as pkg
    return pkg


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def planted(form, d, heads):
    """(cache, columns whose score is infinite): a sequence of twelve full pages of which six have such keys in head 0."""
    c = ref.Cache(d, form, heads, d, PAGE, [PAGE * COLUMNS])
    at = [int(p) for p in c.table[0]]
    if form == "code4":                                      # by the norms: a row's coordinates are all infinite, or no numbers
        n = c.norms[0]
        n[at[1], 0, 5] = INF
        n[at[3], 0, :] = INF
        n[at[5], 0, :] = np.nan                              # the page has no number at all
        n[at[7], 0, 2:9] = np.nan
        n[at[9], 0, 0], n[at[9], 0, 1] = np.nan, INF
        return c, [1, 3, 9]
    k = c.rows16[0]
    k[at[1], 0, 5, 3] = INF                                  # one token
    k[at[2], 0, 6, d - 2] = -INF
    k[at[3], 0, :, 17], k[at[4], 0, :, 40] = INF, -INF       # every token
    k[at[5], 0, :, 9] = np.nan                               # no token has a number there
    k[at[6], 0, :, :] = np.nan
    k[at[7], 0, 3, 7] = np.nan
    k[at[8], 0, 2, 11], k[at[8], 0, 9, 11], k[at[8], 0, 4, 30] = INF, -INF, -INF
    return c, [1, 2, 3, 4, 8]


def score_both(c, q, starts=None):
    """Scores of the last row alone, and of all rows."""
    t, codec = c.device()
    kind = torch.float16 if c.form == "code4" else ref.TYPES[c.form]
    box = torch.full((c.pages, c.heads, 2, c.d), 7.0, dtype=kind, device=DEV)
    _pkg().kv_digest(t["pool"], box, t["table"], t["lengths"], starts=ints([0, c.lens[0]]), **codec)
    rows = q.shape[0]
    one = _pkg().kv_score(q[-1:].contiguous().to(DEV), box, t["pool"], t["table"], t["lengths"], **codec)
    all_ = _pkg().kv_score(q.to(DEV), box, t["pool"], t["table"], t["lengths"], starts=ints([0, rows]), max_new=rows, **codec)
    return box.cpu(), one, all_, t


def finite_box(box):
    """Digests as scores take them: an interval that has no number is 0 to 0; infinite ends, whose pages are looked at apart, are 0 here."""
    box = box.double().clone()
    return torch.where(box.isinf(), 0.0, box)


@pytest.mark.parametrize("d", (64, 96, 128, 192, 256))
@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("group", (1, 3, 4, 16))
def test_infinite_keys_and_keys_that_are_no_numbers(form, kind, d, group):
    heads = 2
    c, high = planted(form, d, heads)
    g = torch.Generator().manual_seed(d + group)
    q = torch.randn(5, heads * group, d, generator=g)
    q[1, :group, [3, 17, 9]] = 0.0                           # nothing meets the coordinate
    q[2, :group] = q[2, :group].abs()                        # one side alone
    q[3, :group] = -q[3, :group].abs()
    q[4, :group, 11] = 0.0
    q = q.to(ref.TYPES[kind])
    print(f"scores {form} {kind} d={d} group={group}", flush=True)
    box, one, all_, t = score_both(c, q)
    want, bound = pick.scores(c, q, finite_box(box), [5])
    want[:, 0, high] = INF
    bound[:, 0, high] = 0.0
    for got, rows in ((one, [4]), (all_, range(5))):
        got, want_, bound_ = got.double().cpu().numpy(), want[list(rows)], bound[list(rows)]
        assert np.array_equal(np.isposinf(got), np.isposinf(want_)) and np.array_equal(np.isneginf(got), np.isneginf(want_))
        fine = np.isfinite(want_)
        assert np.isfinite(got[fine]).all() and (np.abs(got[fine] - want_[fine]) <= bound_[fine]).all()
    a = _pkg().kv_select(one, t["lengths"], PAGE, 7).cpu().numpy()
    b = _pkg().kv_select(all_, t["lengths"], PAGE, 7, starts=ints([0, 5])).cpu().numpy()
    for chosen in (a[0, 0], b[4, 0]):
        assert set(high) <= set(chosen.tolist())             # none of their keys is passed over
    assert np.array_equal(a[0, 0], b[4, 0])


@pytest.mark.parametrize("d", (64, 128, 192))
@pytest.mark.parametrize("form,kind", FORMS)
@pytest.mark.parametrize("group", (1, 3, 8))
def test_queries_that_are_no_finite_numbers(form, kind, d, group):
    """They count for nothing: a coordinate as if it were zero; over codes, where the rotation mixes them, the whole query."""
    heads = 2
    c = ref.Cache(d, form, heads, d, PAGE, [PAGE * COLUMNS])
    q = torch.randn(5, heads * group, d, generator=torch.Generator().manual_seed(d + group)).to(ref.TYPES[kind])
    bad = [(0, 0, 5, np.nan), (1, 0, 7, INF), (1, group, d - 1, -INF), (2, group - 1, 0, np.nan), (4, 0, 3, INF), (4, heads * group - 1, 9, -INF), (4, 0, 8, np.nan)]
    clean = q.clone()
    for r, h, j, v in bad:
        q[r, h, j] = v
        clean[r, h, (slice(None) if form == "code4" else j)] = 0.0
    q[3], clean[3] = np.nan, 0.0                             # nothing of the row is a number
    print(f"queries {form} {kind} d={d} group={group}", flush=True)
    box, one, all_, _ = score_both(c, q)
    _, one_clean, all_clean, _ = score_both(c, clean)
    assert torch.equal(one, one_clean) and torch.equal(all_, all_clean)
    want, bound = pick.scores(c, clean, box, [5])
    for got, rows in ((one, [4]), (all_, range(5))):
        assert (np.abs(got.double().cpu().numpy() - want[list(rows)]) <= bound[list(rows)]).all()


@pytest.mark.parametrize("d", (64, 128, 256))
@pytest.mark.parametrize("form,kind", FORMS)
def test_scores_bound_the_products(form, kind, d):
    """No key of a page has larger products, summed over the group's heads, than its score: in 16 bits to the float32 sums, over codes to half a
    float16 step of every coordinate of the digest besides."""
    heads, group = 2, 3
    c = ref.Cache(d, form, heads, d, PAGE, [PAGE * COLUMNS])
    q = torch.randn(5, heads * group, d, generator=torch.Generator().manual_seed(d)).to(ref.TYPES[kind])
    print(f"bounds {form} {kind} d={d}", flush=True)
    box, one, all_, _ = score_both(c, q)
    _, off = pick.scores(c, q, box, [5])
    size = box.double().abs().amax(2).numpy()                # [pages, heads, d]
    for h in range(heads):
        k = c.rotated(0, 0, h, c.lens[0]).reshape(COLUMNS, PAGE, d)
        for r in range(5):
            z = q[r, h * group: (h + 1) * group].double().numpy()
            if form == "code4":
                z = z @ c.rotation.astype(np.float64).T
            most = np.einsum("gd,ctd->gct", z, k).max(2).sum(0)
            seen = (PAGE * COLUMNS - 5 + r) // PAGE + 1
            # a digest is norm * level in float32 (2^-24) rounded to float16 (2^-11, under 2^-14 2^-25)
            step = np.abs(z).sum(0) @ ((2.0 ** -11 + 2.0 ** -23) * size[c.table[0], h] + 2.0 ** -25).T if form == "code4" else 0.0
            # (the last column's page is whole in its digest, but a row sees a part of it: its score bounds that too)
            for got in (all_[r, h],) + ((one[0, h],) if r == 4 else ()):
                assert (got.double().cpu().numpy()[:seen] >= (most - off[r, h] - step)[:seen]).all()
