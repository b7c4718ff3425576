"""Rows appended to the paged cache and read back, against float64: 16 bits exactly, codes next to every border within what the
rotation's arithmetic allows."""
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


def new_rows(seed, rows, heads, d, dtype):
    g = torch.Generator().manual_seed(seed)
    kv = torch.randn(rows, 2, heads, d, generator=g) * torch.rand(rows, 2, heads, 1, generator=g).mul(4).exp()
    return kv.to(dtype).to(DEV)


CASES = [  # (cache, rows, heads, d, page, tokens before, new tokens)
    ("f16", "f16", 1, 64, 16, [0], [1]),
    ("bf16", "bf16", 3, 96, 16, [5, 0, 31, 16], [1, 40, 0, 17]),
    ("f16", "f16", 8, 128, 64, [0, 63, 64], [200, 1, 65]),
    ("bf16", "bf16", 2, 256, 128, [127, 3], [2, 129]),
    ("code4", "f16", 1, 64, 16, [0], [1]),
    ("code4", "bf16", 3, 96, 16, [5, 0, 31, 16], [1, 40, 0, 17]),
    ("code4", "f16", 8, 128, 64, [0, 63, 64], [200, 1, 65]),
    ("code4", "bf16", 5, 192, 32, [7, 8, 9], [9, 8, 7]),
    ("code4", "bf16", 2, 256, 128, [127, 3], [2, 129]),
]


@pytest.mark.parametrize("form,kind,heads,d,page,past,news", CASES)
@pytest.mark.parametrize("single", (False, True))
def test_append_then_read(form, kind, heads, d, page, past, news, single):
    pkg = _pkg()
    if single:                                          # one row per sequence, without starts
        news = [1] * len(past)
    c = ref.Cache(7 * d + page, form, heads, d, page, [a + b for a, b in zip(past, news)])
    t, codec = c.device()
    before = t["pool"].clone()
    kv = new_rows(d, sum(news), heads, d, ref.TYPES[kind])
    k, v = kv[:, 0], kv[:, 1]                           # rows apart in memory, as a projection leaves them
    where = {} if single else {"starts": starts_of(news)}
    print(f"append {form} d={d} page={page} new={news}", flush=True)
    pkg.kv_append(t["pool"], k, v, t["table"], t["lengths"], **where, **codec)
    torch.cuda.synchronize()
    old = ref.Cache(7 * d + page, form, heads, d, page, c.lens)
    c.take(t["pool"].cpu())
    # what the new rows are, token by token; everything else is as it was
    seq = [b for b, n in enumerate(news) for _ in range(n)]
    pos = [past[b] + i for b, n in enumerate(news) for i in range(n)]
    pages = np.array([c.table[b, p // page] for b, p in zip(seq, pos)])
    inside = np.array(pos) % page
    touched = np.zeros((c.pages, page), bool)
    touched[pages, inside] = True
    if form != "code4":
        for i, x in enumerate((k, v)):
            assert torch.equal(c.rows16[i, pages, :, inside], x.cpu())
        now, was = c.rows16.clone(), old.rows16.clone()
        now.transpose(2, 3)[:, torch.from_numpy(touched)] = 0
        was.transpose(2, 3)[:, torch.from_numpy(touched)] = 0
        assert torch.equal(now, was)
    else:
        assert np.array_equal(c.codes.swapaxes(2, 3)[:, ~touched], old.codes.swapaxes(2, 3)[:, ~touched])
        assert np.array_equal(c.norms.swapaxes(2, 3)[:, ~touched], old.norms.swapaxes(2, 3)[:, ~touched])
        level = c.levels.astype(np.float64)
        border = (level[1:] + level[:-1]) / 2
        for i, x in enumerate((k, v)):
            x = x.double().cpu().numpy()
            norm = np.linalg.norm(x, axis=-1)
            rho = x @ c.rotation.astype(np.float64).T / norm[..., None]
            want = np.searchsorted(border, rho, side="right")
            got = c.codes[i, pages, :, inside]
            far = np.abs(rho[..., None] - border).min(axis=-1) > 2.0 ** -19
            assert np.array_equal(got[far], want[far])
            assert (np.abs(got.astype(int) - want)[~far] <= 1).all()
            g = c.norms[i, pages, :, inside].astype(np.float64)
            assert (np.abs(g - norm) <= norm * (2.0 ** -11 + 2.0 ** -18)).all()
    # and back
    kb, vb = (torch.full((sum(news), heads, d), 7.0, dtype=ref.TYPES[kind], device=DEV) for _ in range(2))
    pkg.kv_read(t["pool"], t["table"], t["lengths"], kb, vb, **where, **codec)
    torch.cuda.synchronize()
    for i, x in enumerate((kb, vb)):
        got = x.double().cpu().numpy()
        if form != "code4":
            assert torch.equal(x.cpu(), c.rows16[i, pages, :, inside])
            continue
        want = level[c.codes[i, pages, :, inside]] * c.norms[i, pages, :, inside, None].astype(np.float64) @ c.rotation.astype(np.float64)
        size = np.linalg.norm(want, axis=-1, keepdims=True)
        assert (np.abs(got - want) <= ref.HALF[x.dtype] * np.abs(want) + 2.0 ** -18 * size + 2.0 ** -25).all()
    assert before.shape == t["pool"].shape


@pytest.mark.parametrize("form", ("bf16", "code4"))
def test_rows_without_a_place(form):
    """Missing pages, pages that are none, lengths of zero, over the table and under the new rows: nothing is written elsewhere, reading gives zeros."""
    pkg = _pkg()
    c = ref.Cache(3, form, 2, 64, 16, [40, 20, 20, 0, 33], columns=4)
    t, codec = c.device()
    table = t["table"].clone()
    table[0, 1], table[0, 2] = -1, c.pages                  # tokens 16 .. 39 of sequence 0 have no page
    lengths = torch.tensor([40, 2, 1000, 0, -5], dtype=torch.int32, device=DEV)   # 1000: over 4 columns, counts as 64 and its tokens have no page
    news = [26, 5, 3, 2, 1]
    kv = new_rows(1, sum(news), 2, 64, torch.bfloat16)
    before = t["pool"].clone()
    pkg.kv_append(t["pool"], kv[:, 0], kv[:, 1], table, lengths, starts=starts_of(news), **codec)
    torch.cuda.synchronize()
    a, b = ref.Cache(3, form, 2, 64, 16, c.lens, columns=4), ref.Cache(3, form, 2, 64, 16, c.lens, columns=4)
    a.take(before.cpu())
    b.take(t["pool"].cpu())
    x, y = (a.codes, b.codes) if form == "code4" else (a.rows16.view(torch.int16).numpy(), b.rows16.view(torch.int16).numpy())
    changed = (x != y).any(axis=(0, 2, 4))                  # [page, token]
    allowed = np.zeros_like(changed)
    allowed[c.table[0, 0], 14:16] = True                    # positions 14 .. 39, of which 14 and 15 have a page
    allowed[c.table[1, 0], :2] = True                       # length 2 with 5 new rows: the last two
    assert not (changed & ~allowed).any() and changed[allowed].all()
    kb, vb = (torch.full((sum(news), 2, 64), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pkg.kv_read(t["pool"], table, lengths, kb, vb, starts=starts_of(news), **codec)
    torch.cuda.synchronize()
    placed = torch.zeros(sum(news), dtype=torch.bool)
    placed[:2] = True
    placed[26 + 3: 26 + 5] = True
    for z in (kb, vb):
        assert (z.cpu()[~placed] == 0).all() and (z.cpu()[placed] != 0).any()


def test_rows_of_zero_and_of_no_number():
    """A row of zeros stands for zeros; a row with a NaN spoils itself alone; so does one whose norm float16 cannot hold."""
    pkg = _pkg()
    d, news = 128, [9]
    c = ref.Cache(5, "code4", 1, d, 16, news)
    t, codec = c.device()
    kv = torch.randn(9, 2, 1, d, generator=torch.Generator().manual_seed(5)).bfloat16().to(DEV)
    kv[2] = 0
    kv[4, :, 0, 3] = float("nan")
    kv[6] = 3e4                                             # norm 3.4e5
    kv[7] *= 1e-30
    pkg.kv_append(t["pool"], kv[:, 0], kv[:, 1], t["table"], t["lengths"], starts=starts_of(news), **codec)
    kb, vb = (torch.empty(9, 1, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pkg.kv_read(t["pool"], t["table"], t["lengths"], kb, vb, starts=starts_of(news), **codec)
    torch.cuda.synchronize()
    for x, y in ((kb, kv[:, 0]), (vb, kv[:, 1])):
        x, y = x.float().cpu(), y.float().cpu()
        assert (x[2] == 0).all() and (x[7].abs() < 1e-6).all()
        assert not torch.isfinite(x[4]).all() and not torch.isfinite(x[6]).any()
        good = [0, 1, 3, 5, 8]
        # the others: the nearest levels of the rotated row, wherever no coordinate stands next to a border
        level, turn = c.levels.astype(np.float64), c.rotation.astype(np.float64)
        border = (level[1:] + level[:-1]) / 2
        for i in good:
            row = y[i, 0].double().numpy()
            norm = np.linalg.norm(row)
            rho = turn @ row / norm
            if np.abs(rho[:, None] - border).min() <= 2.0 ** -19:
                continue
            want = level[np.searchsorted(border, rho, side="right")] @ turn * float(np.float16(norm))
            assert (np.abs(x[i, 0].double().numpy() - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -18 + 2.0 ** -11) * norm).all()


def test_other_stream_and_strides():
    pkg = _pkg()
    c = ref.Cache(9, "code4", 2, 64, 32, [50, 3])
    t, codec = c.device()
    wide = torch.full((2, 9), -1, dtype=torch.int32, device=DEV)
    wide[:, : c.columns] = t["table"]
    kv = new_rows(4, 2, 2, 64, torch.float16)
    one, two = t["pool"].clone(), t["pool"].clone()
    pkg.kv_append(one, kv[:, 0].contiguous(), kv[:, 1].contiguous(), t["table"], t["lengths"], **codec)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    pkg.kv_append(two, kv[:, 0], kv[:, 1], wide[:, : c.columns], t["lengths"], stream=s, **codec)
    torch.cuda.synchronize()
    assert torch.equal(one, two)


@pytest.mark.parametrize("kind,scale", [("f16", 2.0 ** -17), ("f16", 1000.0), ("bf16", 2.0 ** -100), ("bf16", 2.0 ** 9), ("bf16", 2.0 ** -17)])
@pytest.mark.parametrize("single", (False, True))
def test_codes_of_short_and_long_rows(kind, scale, single):
    """Codes depend on a row's direction alone: rows of subnormal float16 numbers, rows near the largest norm, rows far under it."""
    pkg = _pkg()
    d, n = 128, 40
    lens = [1] * n if single else [n]
    c = ref.Cache(12, "code4", 1, d, 16, lens)
    t, codec = c.device()
    x = (torch.randn(n, 2, 1, d, generator=torch.Generator().manual_seed(9)) * scale).to(ref.TYPES[kind])
    where = {} if single else {"starts": starts_of([n])}
    pkg.kv_append(t["pool"], x[:, 0].to(DEV), x[:, 1].to(DEV), t["table"], t["lengths"], **where, **codec)
    torch.cuda.synchronize()
    c.take(t["pool"].cpu())
    level = c.levels.astype(np.float64)
    border = (level[1:] + level[:-1]) / 2
    seq, pos = (range(n), [0] * n) if single else ([0] * n, range(n))
    pages, inside = [c.table[b, p // 16] for b, p in zip(seq, pos)], [p % 16 for p in pos]
    for i in range(2):
        rows = x[:, i, 0].double().numpy()
        norm = np.linalg.norm(rows, axis=-1)
        if norm.max() < 2.0 ** -63:                          # shorter than float32 can square: zeros
            assert (c.norms[i, pages, 0, inside] == 0).all()
            continue
        rho = rows @ c.rotation.astype(np.float64).T / norm[:, None]
        far = np.abs(rho[..., None] - border).min(axis=-1) > 2.0 ** -19
        assert np.array_equal(c.codes[i, pages, 0, inside][far], np.searchsorted(border, rho, side="right")[far])
        got = c.norms[i, pages, 0, inside].astype(np.float64)
        assert (np.abs(got - norm) <= norm * (2.0 ** -11 + 2.0 ** -18) + 2.0 ** -25).all()
