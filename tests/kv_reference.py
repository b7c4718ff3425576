"""The paged key-value cache in float64 on the CPU, written from its definition: pools made and read element by element of the
documented layout, attention row by row.  Also what a result may be off by."""
import math

import numpy as np
import torch

HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}          # most that one rounding moves a value, relative
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


class Cache:
    """A cache with pages scattered over its pool, its content in float64, and the device tensors to call with."""

    def __init__(self, seed, form, heads, d, page, lens, spare=3, columns=None, fill=None, shared=None):
        import paper_2605_17415_amd as pkg
        self.form, self.heads, self.d, self.page, self.lens = form, heads, d, page, list(lens)
        self.rng = np.random.default_rng(seed)
        need = [-(-n // page) for n in lens]
        self.columns = columns or max(max(need, default=1), 1)
        self.pages = sum(need) + spare
        order = self.rng.permutation(self.pages)
        self.table = np.full((len(lens), self.columns), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at: at + n]
            at += n
        self.rotation = self.levels = None
        if form == "code4":
            self.rotation = pkg.ivftq_haar_rotation(d, seed + 1)
            self.levels = pkg.ivftq_build_codebook(4, d)[0]
            self.codes = self.rng.integers(0, 16, (2, self.pages, heads, page, d)).astype(np.uint8)       # ascending order, 0 .. 15
            self.norms = (self.rng.uniform(0.2, 3.0, (2, self.pages, heads, page)) * math.sqrt(d)).astype(np.float16)
        else:
            self.rows16 = torch.from_numpy(self.rng.standard_normal((2, self.pages, heads, page, d))).to(TYPES[form])

    # -- layout
    def pool(self):
        p, h, page, d = self.pages, self.heads, self.page, self.d
        if self.form != "code4":
            k, v = self.rows16
            out = torch.empty(p, h, 2, page, d, dtype=k.dtype)
            out[:, :, 0] = k
            out[:, :, 1] = v.reshape(p, h, page // 8, 8, d).transpose(3, 4).reshape(p, h, page, d)
            return out
        nib = np.where(self.codes >= 8, self.codes - 8, 15 - self.codes).astype(np.uint8)
        k = nib[0]
        v = nib[1].reshape(p, h, page // 8, 8, d).swapaxes(3, 4)
        parts = [(x[..., 0::2] | x[..., 1::2] << 4).reshape(p, h, -1) for x in (k, v)]
        parts += [x.view(np.uint8).reshape(p, h, -1) for x in self.norms]
        return torch.from_numpy(np.concatenate(parts, axis=-1))

    def take(self, pool):
        """Content from a pool (the opposite of pool())."""
        p, h, page, d = self.pages, self.heads, self.page, self.d
        if self.form != "code4":
            self.rows16 = torch.stack([pool[:, :, 0], pool[:, :, 1].reshape(p, h, page // 8, d, 8).transpose(3, 4).reshape(p, h, page, d)])
            return
        raw = pool.numpy()
        half = page * d // 2
        nib = [np.stack([x & 15, x >> 4], -1).reshape(p, h, -1) for x in (raw[..., :half], raw[..., half: 2 * half])]
        nib = np.stack([nib[0].reshape(p, h, page, d), nib[1].reshape(p, h, page // 8, d, 8).swapaxes(3, 4).reshape(p, h, page, d)])
        self.codes = np.where(nib >= 8, 15 - nib, nib + 8).astype(np.uint8)
        n = np.ascontiguousarray(raw[..., 2 * half:]).view(np.float16)
        self.norms = np.stack([n[..., :page], n[..., page:]])

    def device(self, dev="cuda:0"):
        t = {"pool": self.pool().to(dev), "table": torch.from_numpy(self.table).to(dev), "lengths": torch.tensor(self.lens, dtype=torch.int32, device=dev)}
        codec = {"rotation": torch.from_numpy(self.rotation).to(dev), "levels": self.levels} if self.form == "code4" else {}
        return t, codec

    # -- content
    def rotated(self, kind, b, h, n):
        """Keys (0) or values (1) of the first n tokens in the frame they are stored in, float64; NaN where a page is missing."""
        out = np.full((n, self.d), np.nan)
        for t0 in range(0, n, self.page):
            col = t0 // self.page
            page = self.table[b, col] if col < self.columns else -1
            if not 0 <= page < self.pages:
                continue
            m = min(self.page, n - t0)
            if self.form == "code4":
                out[t0: t0 + m] = self.levels.astype(np.float64)[self.codes[kind, page, h, :m]] * self.norms[kind, page, h, :m, None].astype(np.float64)
            else:
                out[t0: t0 + m] = self.rows16[kind, page, h, :m].double().numpy()
        return out

    def rows(self, kind, b, h, n):
        x = self.rotated(kind, b, h, n)
        return x @ self.rotation.astype(np.float64) if self.form == "code4" else x


def attention(cache, q, news, window=0, sinks=0, scale=None, max_new=None):
    """(out, lse, bound, norm): results of every row, float64 [rows, heads, d]; how far each coordinate may be off, from the
    roundings of the kernels; for codes how far the whole row may be off (2-norm) before the output's own rounding."""
    d, kv, group = cache.d, cache.heads, q.shape[1] // cache.heads
    scale = 1 / math.sqrt(d) if scale is None else scale
    step = HALF[q.dtype]
    x = q.double().numpy()
    out, lse = np.zeros(x.shape), np.full(x.shape[:2], -np.inf)
    bound, norm = np.zeros(x.shape), np.zeros(x.shape[:2])
    row = 0
    for b, (n, new) in enumerate(zip(cache.lens, news)):
        for h in range(kv):
            k, v = cache.rows(0, b, h, n), cache.rows(1, b, h, n)
            there = ~np.isnan(cache.rotated(0, b, h, n)).all(axis=1) if n else np.zeros(0, bool)
            for i in range(new):
                p = n - new + i
                t = np.arange(n)
                seen = there & (t <= p)
                if window:
                    seen &= (t > p - window) | (t < sinks)
                if not seen.any():
                    continue
                for g in range(group):
                    r, hq = row + i, h * group + g
                    s = scale * (k[seen] @ x[r, hq])
                    w = np.exp(s - s.max())
                    total = w.sum()
                    out[r, hq] = w @ v[seen] / total
                    lse[r, hq] = s.max() + np.log(total)
                    size = w @ np.abs(v[seen]) / total
                    # a score's float32 sum of d products, its product with the scale and the exponent's argument
                    off = (d + 4) * 2.0 ** -24 * np.max(scale * (np.abs(k[seen]) @ np.abs(x[r, hq]))) + 4 * 2.0 ** -24 * np.abs(s).max()
                    if cache.form != "code4":
                        # weights rounded to the type once (float16: not under 2^-25 in absolute terms), sums in float32
                        tiny = 2.0 ** -25 * np.abs(v[seen]).sum(axis=0) / total if q.dtype == torch.float16 else 0.0
                        bound[r, hq] = (step + 2 * off + (n + 40) * 2.0 ** -24) * size + tiny + step * np.abs(out[r, hq])
                    else:
                        # the rotated unit query and the levels rounded to float16: 2^-11 each, of every product
                        z = cache.rotation.astype(np.float64) @ x[r, hq]
                        kr, vr = cache.rotated(0, b, h, n)[seen], cache.rotated(1, b, h, n)[seen]
                        off += 2 * 2.0 ** -11 * np.max(scale * (np.abs(kr) @ np.abs(z))) + 2.0 ** -20 * np.max(scale * np.abs(kr).sum(axis=1)) * np.linalg.norm(z)
                        # weights times norms and the values' levels the same
                        length = np.linalg.norm(vr, axis=1)
                        norm[r, hq] = (np.expm1(2 * off) + 2 * 2.0 ** -11 + (n + 40) * 2.0 ** -24 + 2.0 ** -19) * (w @ length) / total
                        norm[r, hq] += 2.0 ** -25 * np.linalg.norm(vr / np.maximum(cache_norms(cache, b, h, n)[seen][:, None], 1e-30), axis=1).sum() / total
        row += new
    return out, lse, bound, norm


def cache_norms(cache, b, h, n):
    out = np.ones(n)
    for t0 in range(0, n, cache.page):
        page = cache.table[b, t0 // cache.page]
        if 0 <= page < cache.pages:
            m = min(cache.page, n - t0)
            out[t0: t0 + m] = cache.norms[1, page, h, :m].astype(np.float64)
    return out


def check_attention(cache, q, got, news, lse=None, **mask):
    out, logs, bound, norm = attention(cache, q, news, **mask)
    x = got.double().cpu().numpy()
    assert np.isfinite(x).all()
    diff = np.abs(x - out)
    if cache.form == "code4":
        rounding = HALF[q.dtype] * (np.abs(out) + diff) + 2.0 ** -25
        off = np.linalg.norm(np.maximum(diff - rounding, 0), axis=-1)
        assert (off <= norm + 1e-12).all(), f"row off by {np.max(off / np.maximum(norm, 1e-30)):.3g} of what it may be"
    else:
        ratio = diff / np.maximum(bound + 2.0 ** -25, 1e-30)
        assert (ratio <= 1).all(), f"coordinate off by {ratio.max():.3g} of what it may be"
    if lse is not None:
        y = lse.double().cpu().numpy()
        empty = np.isneginf(logs)
        assert np.array_equal(np.isneginf(y), empty)
        assert not empty.any() or (x[empty] == 0).all()
        far = np.abs(y - logs)[~empty]
        assert (far <= (2e-2 if cache.form == "code4" else 1e-4)).all(), far.max()
