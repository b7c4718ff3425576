"""Digests, scores, chosen pages and attention over them in float64 on the CPU, from their definitions.  Also what a result may be off by."""
import math

import numpy as np

from kv_reference import HALF, cache_norms


def keys_as_stored(cache, page, h, tokens):
    """Keys of a page's first tokens as a digest has them: 16 bits as they are, codes level * norm in float32, rounded to float16."""
    if cache.form != "code4":
        return cache.rows16[0, page, h, :tokens].double().numpy()
    product = cache.levels[cache.codes[0, page, h, :tokens]] * cache.norms[0, page, h, :tokens, None].astype(np.float32)
    return product.astype(np.float16).astype(np.float64)


def digests(cache):
    """{page: [heads, 2, d]} of every page that a sequence has tokens in."""
    out = {}
    for b, n in enumerate(cache.lens):
        for col in range(-(-n // cache.page)):
            page = cache.table[b, col] if col < cache.columns else -1
            if 0 <= page < cache.pages:
                k = [keys_as_stored(cache, page, h, min(cache.page, n - col * cache.page)) for h in range(cache.heads)]
                with np.errstate(invalid="ignore"):
                    out[int(page)] = np.stack([np.stack([np.fmin.reduce(x, 0, initial=np.inf), np.fmax.reduce(x, 0, initial=-np.inf)]) for x in k])
    return out


def positions(lens, news):
    """(sequence, position) of every new row."""
    return [(b, n - m + i) for b, (n, m) in enumerate(zip(lens, news)) for i in range(m)]


def scores(cache, q, box, news):
    """(scores, how far they may be off) [rows, heads, columns]; box: digests [pages, heads, 2, d]."""
    x, box = q.double().cpu().numpy(), box.double().cpu().numpy()
    heads, d, group = cache.heads, cache.d, q.shape[1] // cache.heads
    out = np.full((x.shape[0], heads, cache.columns), -np.inf)
    bound = np.zeros(out.shape)
    for r, (b, p) in enumerate(positions(cache.lens, news)):
        for col in range(cache.columns):
            page = cache.table[b, col]
            if p < 0 or col * cache.page > p or not 0 <= page < cache.pages:
                continue
            for h in range(heads):
                z = x[r, h * group: (h + 1) * group]
                low, high = box[page, h]
                size = np.maximum(np.abs(low), np.abs(high))
                if cache.form == "code4":
                    z = z @ cache.rotation.astype(np.float64).T
                    # rotated rows are good to 2^-21 of their length a coordinate, and go in as two float16 parts
                    bound[r, h, col] += 2.0 ** -20 * np.linalg.norm(z, axis=1).sum() * size.sum()
                terms = np.maximum(z * low, z * high)
                out[r, h, col] = terms.sum()
                # float32 sums of 2 d products a query head, each addition off by a unit in the last place of what it adds up to at most
                bound[r, h, col] += (2 * d * group + 8) * 2.0 ** -23 * (np.abs(z) * size).sum()
    return out, bound


def select(scores, lens, news, page, count, first, last):
    """[rows, heads, count] from scores as float32."""
    rows, heads, columns = scores.shape
    out = np.full((rows, heads, count), -1, np.int32)
    for r, (_, p) in enumerate(positions(lens, news)):
        n = min(p // page + 1, columns) if p >= 0 else 0
        for h in range(heads):
            kept = [c for c in range(n) if c < first or c >= n - last]
            rest = [c for c in range(n) if c not in set(kept) and scores[r, h, c] > -np.inf]
            rest.sort(key=lambda c: (-float(scores[r, h, c]), c))
            got = sorted(kept + rest[: count - len(kept)])[:count]
            out[r, h, : len(got)] = got
    return out


def listed(entries):
    """The entries that count: those above every one before them."""
    out, top = [], -1
    for e in entries:
        if e > top:
            out.append(int(e))
            top = e
    return out


def check_attention(cache, q, got, news, chosen, lse=None, scale=None):
    """Results over chosen pages against float64; the roundings that may be between them are those of attention over the whole cache."""
    d, kv, group = cache.d, cache.heads, q.shape[1] // cache.heads
    scale = 1 / math.sqrt(d) if scale is None else scale
    step, x = HALF[q.dtype], q.double().numpy()
    y, logs = got.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    for r, (b, p) in enumerate(positions(cache.lens, news)):
        n = cache.lens[b]
        for h in range(kv):
            k, v = cache.rows(0, b, h, n), cache.rows(1, b, h, n)
            there = ~np.isnan(cache.rotated(0, b, h, n)).all(axis=1) if n else np.zeros(0, bool)
            t = np.arange(n)
            seen = there & (t <= p) & np.isin(t // cache.page, listed(chosen[r, h]))
            for g in range(group):
                hq = h * group + g
                if not seen.any():
                    assert (y[r, hq] == 0).all()
                    assert logs is None or logs[r, hq] == -np.inf
                    continue
                s = scale * (k[seen] @ x[r, hq])
                w = np.exp(s - s.max())
                total = w.sum()
                out = w @ v[seen] / total
                off = (d + 4) * 2.0 ** -24 * np.max(abs(scale) * (np.abs(k[seen]) @ np.abs(x[r, hq]))) + 4 * 2.0 ** -24 * np.abs(s).max()
                diff = np.abs(y[r, hq] - out)
                assert np.isfinite(diff).all()
                if cache.form != "code4":
                    # weights rounded to the type once (float16: not under 2^-25 in absolute terms), sums in float32
                    tiny = 2.0 ** -25 * np.abs(v[seen]).sum(axis=0) / total if step == 2.0 ** -11 else 0.0
                    bound = (step + 2 * off + (n + 40) * 2.0 ** -24) * (w @ np.abs(v[seen]) / total) + tiny + step * np.abs(out) + 2.0 ** -25
                    assert (diff <= bound).all(), f"row {r} head {hq}: off by {(diff / bound).max():.3g} of what it may be"
                else:
                    # the rotated unit query and the levels rounded to float16, weights times norms and the values' levels the same
                    z = cache.rotation.astype(np.float64) @ x[r, hq]
                    kr, vr = cache.rotated(0, b, h, n)[seen], cache.rotated(1, b, h, n)[seen]
                    off += 2 * 2.0 ** -11 * np.max(abs(scale) * (np.abs(kr) @ np.abs(z))) + 2.0 ** -20 * np.max(abs(scale) * np.abs(kr).sum(axis=1)) * np.linalg.norm(z)
                    length = np.linalg.norm(vr, axis=1)
                    norm = (np.expm1(2 * off) + 2 * 2.0 ** -11 + (n + 40) * 2.0 ** -24 + 2.0 ** -19) * (w @ length) / total
                    norm += 2.0 ** -25 * np.linalg.norm(vr / np.maximum(cache_norms(cache, b, h, n)[seen][:, None], 1e-30), axis=1).sum() / total
                    rounding = step * (np.abs(out) + diff) + 2.0 ** -25
                    far = np.linalg.norm(np.maximum(diff - rounding, 0))
                    assert far <= norm + 1e-12, f"row {r} head {hq}: off by {far / norm:.3g} of what it may be"
                if logs is not None:
                    assert abs(logs[r, hq] - (s.max() + np.log(total))) <= off + 2.0 ** -18 * (1 + abs(s.max())) + (n + 40) * 2.0 ** -24
