"""The paged key-value cache whose speed is measured: rows appended to it, attention that reads it, its pages managed.

A server that answers with a language model keeps the keys and values of every token in pages, either in 16 bits or in
the 4-bit codes of this library (fixed rotation, Lloyd-Max levels, a float16 norm for each row).  Each step it appends
the new tokens, attends from them to what is visible in the cache, and forks, frees and compacts pages.

Layout of one page of one key-value head, tokens t < page, coordinates j < d:
  16 bits   K[t][j], then V[t / 8][j][t % 8]
  codes     the same two blocks in 4 bits (low half of a byte first; bit 3 = sign, bits 0-2 = magnitude, level[8 + m] or
            -level[8 + m]), then float16 norms of the keys and of the values; coordinates are those of the rotated row
`own` false: elementary torch operations; true: the library's entry points.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # a decoding step of 32 conversations: one row each into a coded cache (latency)
        {"name": "append_step", "op": "append", "cache": "code4", "type": "bf16", "batch": 32, "new": 1, "past": 900, "heads": 8, "d": 128, "page": 64},
        # prompts of a batch as they arrive, ragged, into a coded cache
        {"name": "append_prompts", "op": "append", "cache": "code4", "type": "f16", "batch": 13, "new": 6000, "past": 0, "heads": 8, "d": 128, "page": 64},
        # the same into 16 bits, rows of 96 coordinates, after a shared beginning
        {"name": "append_plain", "op": "append", "cache": "bf16", "type": "bf16", "batch": 7, "new": 4001, "past": 333, "heads": 4, "d": 96, "page": 16},
        # one short conversation, one token: latency alone
        {"name": "token_short", "op": "attend", "cache": "f16", "type": "f16", "batch": 1, "new": 1, "past": 36, "heads": 4, "group": 2, "d": 64, "page": 16,
         "window": 0, "sinks": 0},
        # a served batch of unequal conversations, 16-bit cache
        {"name": "token_batch", "op": "attend", "cache": "bf16", "type": "bf16", "batch": 48, "new": 1, "past": 9000, "heads": 8, "group": 4, "d": 128, "page": 64,
         "window": 0, "sinks": 0},
        # a few very long documents in codes, as a retrieval model's answer reads them
        {"name": "token_long_codes", "op": "attend", "cache": "code4", "type": "bf16", "batch": 4, "new": 1, "past": 131_000, "heads": 8, "group": 8, "d": 128,
         "page": 64, "window": 0, "sinks": 0},
        # a batch in codes with a window and four first tokens, no groups
        {"name": "token_window_codes", "op": "attend", "cache": "code4", "type": "f16", "batch": 61, "new": 1, "past": 7000, "heads": 12, "group": 1, "d": 64,
         "page": 32, "window": 2048, "sinks": 4},
        # ragged prompts with nothing before them
        {"name": "prompts_ragged", "op": "attend", "cache": "f16", "type": "f16", "batch": 5, "new": 1777, "past": 0, "heads": 16, "group": 1, "d": 64, "page": 16,
         "window": 0, "sinks": 0},
        # one long prompt with a window and first tokens that stay visible
        {"name": "prompt_window", "op": "attend", "cache": "bf16", "type": "bf16", "batch": 1, "new": 8192, "past": 0, "heads": 8, "group": 4, "d": 128, "page": 64,
         "window": 4096, "sinks": 4},
        # a chunk of a prompt against a long beginning that is held in codes
        {"name": "chunk_codes", "op": "attend", "cache": "code4", "type": "bf16", "batch": 2, "new": 512, "past": 20_000, "heads": 8, "group": 4, "d": 128, "page": 64,
         "window": 0, "sinks": 0},
        # a scheduler's turn: conversations freed, others forked (beam or shared prompt), pages reserved for what comes
        {"name": "pages_turn", "op": "turn", "batch": 96, "past": 4000, "page": 64, "layers": 4, "record": 16_384, "forks": 24, "frees": 16, "new": 40},
        # a pool brought together after many conversations have ended
        {"name": "pages_compact", "op": "compact", "batch": 64, "past": 8000, "page": 64, "layers": 8, "record": 32_768, "frees": 33},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


#: Most that a drawn case may cost: multiplications and additions of `work`, bytes of `work`, values of the padded score matrix of the plain form.
MOST_FLOPS, MOST_BYTES, MOST_SCORES = 8.2e11, 2.1e9, 2.2e9


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        padded = case["batch"] * case["heads"] * case["group"] * case["new"] * (case["past"] + case["new"]) if case["op"] == "attend" else 0
        gathered = case["batch"] * case["heads"] * (case["past"] + case["new"]) * case["d"] if case["op"] == "attend" else 0
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and padded <= MOST_SCORES and gathered <= 6e8:
            return case


def _draw(rng):
    kind = rng.choice(["append", "few", "few", "many", "many", "pages"])
    page, d = rng.choice([16, 32, 64, 128]), rng.choice([64, 96, 128, 128, 256])
    cache = rng.choice(["f16", "bf16", "code4", "code4"])
    base = {"cache": cache, "type": rng.choice(["f16", "bf16"]) if cache == "code4" else cache, "heads": rng.choice([1, 2, 3, 4, 8, 12, 16]), "d": d, "page": page}
    if kind == "append":
        new = rng.choice([1, _log(rng, 2, 8000)])
        return {"op": "append", **base, "batch": _log(rng, 1, 256 if new == 1 else 24), "new": new, "past": rng.choice([0, _log(rng, 1, 3000)])}
    if kind == "pages":
        batch = _log(rng, 4, 192)
        pages = {"batch": batch, "past": _log(rng, 100, 8000), "page": page, "layers": rng.choice([1, 2, 4, 8]), "record": rng.choice([4096, 8448, 16_384, 32_768])}
        if rng.random() < 0.5:
            return {"op": "turn", **pages, "forks": rng.randint(1, batch // 4), "frees": rng.randint(1, batch // 4), "new": _log(rng, 1, 500)}
        return {"op": "compact", **pages, "frees": rng.randint(1, batch - 1)}
    mask = {"window": 0, "sinks": 0} if rng.random() < 0.5 else {"window": _log(rng, 64, 5000), "sinks": rng.choice([0, 1, 4, 17])}
    base["group"] = rng.choice([1, 2, 3, 4, 5, 8, 16])
    if kind == "few":
        return {"op": "attend", **base, **mask, "batch": _log(rng, 1, 96), "new": 1, "past": _log(rng, 1, 130_000)}
    return {"op": "attend", **base, **mask, "batch": _log(rng, 1, 8), "new": _log(rng, 2, 8000), "past": rng.choice([0, _log(rng, 1, 20_000)])}


def _sizes(case):
    """(tokens in the cache with the new ones, new tokens) of each sequence: fixed by the case, unequal where there are several."""
    r = random.Random("%(batch)d %(past)d %(new)d" % case)
    lens, news = [], []
    for b in range(case["batch"]):
        past = case["past"] if b == 0 else int(round(case["past"] * r.uniform(0.1, 1.0)))
        new = case["new"] if b == 0 else max(1, int(round(case["new"] * r.uniform(0.2, 1.0))))
        lens.append(past + new)
        news.append(new)
    return lens, news


def _visible(length, new, window, sinks):
    """(pairs of a new token and a token visible to it, tokens visible to any)."""
    pos = np.arange(length - new, length, dtype=np.int64)
    if not window:
        return int((pos + 1).sum()), length
    low = np.maximum(pos - window + 1, 0)
    pairs = int((pos + 1 - low + np.minimum(low, sinks)).sum())
    first = max(length - new - window + 1, 0)
    return pairs, length - first + min(first, sinks)


def _row_bytes(case):
    return case["d"] // 2 + 2 if case["cache"] == "code4" else 2 * case["d"]


def work(case):
    if case["op"] == "append":  # rows read, records written, and rows read back from them
        rows = sum(_sizes(case)[1]) * case["heads"]
        spun = 2 * 2 * 2 * rows * case["d"] ** 2 if case["cache"] == "code4" else 0
        return {"bytes": 2 * rows * (4 * case["d"] + 2 * _row_bytes(case)), "flops": spun or rows}
    if case["op"] == "attend":
        lens, news = _sizes(case)
        seen = [_visible(n, m, case["window"], case["sinks"]) for n, m in zip(lens, news)]
        rows = sum(news) * case["heads"] * case["group"]
        flops = 4 * case["d"] * case["heads"] * case["group"] * sum(p for p, _ in seen)
        if case["cache"] == "code4":
            flops += 2 * 2 * rows * case["d"] ** 2
        return {"bytes": 4 * rows * case["d"] + 2 * _row_bytes(case) * case["heads"] * sum(u for _, u in seen), "flops": flops}
    lens, pages = _page_plan(case)
    entries = 4 * (case["batch"] + case.get("forks", 0)) * _columns(case) + 4 * _pool_pages(case)
    if case["op"] == "turn":
        partial = sum(lens[p] % case["page"] != 0 for p in _turn(case)[0])
        return {"bytes": 2 * partial * case["layers"] * case["record"] + 2 * entries, "flops": entries}
    kept = sum(pages[case["frees"]:])
    high = int((_compact_used(case) >= kept).sum())
    return {"bytes": 2 * high * case["layers"] * case["record"] + 2 * entries, "flops": entries}


# ---------------------------------------------------------------------------------------------------- inputs

def _rng(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _levels(d):
    """16 levels for coordinates of a unit row of d: Lloyd's iteration for a normal density of variance 1 / d, symmetric."""
    x = np.linspace(0, 5, 20_001)
    w = np.exp(-x * x / 2)
    c = np.linspace(0.13, 2.7, 8)
    for _ in range(300):
        bin_ = np.searchsorted((c[1:] + c[:-1]) / 2, x, side="right")
        c = np.bincount(bin_, w * x, 8) / np.bincount(bin_, w, 8)
    c = (c / math.sqrt(d)).astype(np.float32)
    return np.concatenate([-c[::-1], c])


def _rotation(d, seed):
    q, r = np.linalg.qr(np.random.RandomState(seed % (1 << 31)).standard_normal((d, d)))
    return torch.from_numpy((q * np.sign(np.diag(r))).astype(np.float32)).to(DEV)


def _bins(levels):
    return torch.from_numpy(((levels[1:].astype(np.float64) + levels[:-1]) / 2)).to(DEV)


def _nibbles(x, levels):
    """Sign and magnitude of the level next to each coordinate."""
    c = torch.bucketize(x, _bins(levels).to(x.dtype), right=True, out_int32=True)
    return torch.where(c >= 8, c - 8, 15 - c).to(torch.uint8)


def _eights(x):
    """[..., page, d] -> [..., page / 8, d, 8], and back by the same exchange."""
    return x.unflatten(-2, (x.shape[-2] // 8, 8)).transpose(-1, -2)


def _bytes(nibbles):
    return nibbles[..., 0::2] | nibbles[..., 1::2] << 4


def _tables(case, lens, seed):
    """Pages of the sequences, scattered over the pool; entries past a sequence's end are -1."""
    page = case["page"]
    need = torch.tensor([-(-n // page) for n in lens], device=DEV)
    columns = int(max(-(-n // page) for n in lens))
    used = int(sum(-(-n // page) for n in lens))
    pool = used + max(2, used // 16)
    order = torch.randperm(pool, generator=_rng(seed), device=DEV)
    at = torch.arange(columns, device=DEV)[None]
    table = torch.where(at < need[:, None], order[(need.cumsum(0) - need)[:, None].add(at).clamp(max=pool - 1)], -1)
    return table.to(torch.int32).contiguous(), pool


def _pool(case, pages, levels, seed):
    """A pool as earlier steps have left it: rows of unequal length."""
    g, h, page, d = _rng(seed + 1), case["heads"], case["page"], case["d"]
    if case["cache"] != "code4":
        return torch.randn(pages, h, 2, page, d, generator=g, device=DEV, dtype=TYPES[case["cache"]])
    parts, norms = [], []
    for value in (False, True):
        x = torch.randn(pages, h, page, d, generator=g, device=DEV)
        n = x.norm(dim=-1, keepdim=True)
        nib = _nibbles(x / n, levels)
        parts.append(_bytes(_eights(nib) if value else nib).reshape(pages, h, -1))
        norms.append((n[..., 0] * (0.5 + torch.rand(pages, h, page, generator=g, device=DEV))).half().view(torch.uint8).reshape(pages, h, -1))
        del x, nib
    return torch.cat(parts + norms, dim=-1)


def _starts(news):
    return torch.tensor([0] + list(np.cumsum(news)), dtype=torch.int32, device=DEV)


def prepare(case, seed):
    if case["op"] in ("turn", "compact"):
        return _prepare_pages(case, seed)
    lens, news = _sizes(case)
    g, t = _rng(seed + 2), TYPES[case["type"]]
    table, pages = _tables(case, lens, seed)
    s = {"case": case, "table": table, "lengths": torch.tensor(lens, dtype=torch.int32, device=DEV), "starts": _starts(news) if case["new"] > 1 else None,
         "longest": max(lens), "most_new": max(news), "rotation": None, "levels": None}
    if case["cache"] == "code4":
        s["rotation"], s["levels"] = _rotation(case["d"], seed), _levels(case["d"])
    rows, h, d = sum(news), case["heads"], case["d"]
    if case["op"] == "append":
        blank = (pages, h, 2, case["page"], d) if case["cache"] != "code4" else (pages, h, case["page"] * (d + 4))
        s["pool"] = torch.zeros(blank, dtype=TYPES.get(case["cache"], torch.uint8), device=DEV)
        # keys and values as a projection gives them: side by side in one matrix, keys with a common part
        kv = torch.randn(rows, 2, h, d, generator=g, device=DEV)
        kv[:, 0] += 0.5 * torch.randn(h, d, generator=g, device=DEV)
        kv = kv.to(t)
        s["k"], s["v"] = kv[:, 0], kv[:, 1]
        s["k_back"], s["v_back"] = torch.empty(rows, h, d, dtype=t, device=DEV), torch.empty(rows, h, d, dtype=t, device=DEV)
    else:
        s["pool"] = _pool(case, pages, s["levels"], seed)
        s["q"] = torch.randn(rows, h * case["group"], d, generator=g, device=DEV, dtype=t)
    return s


# ---------------------------------------------------------------------------------------------------- rows and attention

def _sign_magnitude(levels):
    return torch.from_numpy(np.concatenate([levels[8:], -levels[8:]])).to(DEV)


def _unpack(codes, levels):
    return _sign_magnitude(levels)[torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).int()]


def _stored(s, pages):
    """Keys and values (rotated ones where the cache holds codes) of the given pages, [*pages.shape, heads, page, d] in float32."""
    page, d, h = s["case"]["page"], s["case"]["d"], s["case"]["heads"]
    got = s["pool"][pages]
    if s["case"]["cache"] != "code4":
        k, v = got[..., 0, :, :].float(), got[..., 1, :, :].float()
        return k, v.reshape(*pages.shape, h, page // 8, d, 8).transpose(-1, -2).reshape(*pages.shape, h, page, d)
    half = page * d // 2
    norms = got[..., 2 * half:].contiguous().view(torch.float16).float()
    k = _unpack(got[..., :half], s["levels"]).reshape(*pages.shape, h, page, d)
    v = _unpack(got[..., half:2 * half], s["levels"]).reshape(*pages.shape, h, page // 8, d, 8).transpose(-1, -2).reshape(*pages.shape, h, page, d)
    return k * norms[..., :page, None], v * norms[..., page:, None]


def _places(s):
    """Sequence and position of each new row."""
    rows = (s["k"] if "k" in s else s["q"]).shape[0]
    at = torch.arange(rows, device=DEV)
    if s["starts"] is None:
        return at, s["lengths"].long() - 1, at * 0
    starts = s["starts"].long()
    seq = torch.searchsorted(starts, at, right=True) - 1
    inside = at - starts[seq]
    return seq, s["lengths"].long()[seq] - (starts[1:] - starts[:-1])[seq] + inside, inside


def _plain_append(s):
    page, d, h = s["case"]["page"], s["case"]["d"], s["case"]["heads"]
    seq, pos, _ = _places(s)
    p, t = s["table"].long()[seq, pos // page], pos % page
    if s["case"]["cache"] != "code4":
        s["pool"][p, :, 0, t] = s["k"]
        s["pool"].select(2, 1).view(-1, h, page // 8, d, 8)[p, :, t // 8, :, t % 8] = s["v"]
        return {"k": s["pool"][p, :, 0, t], "v": s["pool"].select(2, 1).view(-1, h, page // 8, d, 8)[p, :, t // 8, :, t % 8]}
    half = page * d // 2
    k_codes = s["pool"][..., :half].view(-1, h, page, d // 2)
    # values: the four bytes of a coordinate's eight tokens as one number, so that a row's half byte can be exchanged
    v_bytes = s["pool"][..., half:2 * half].unflatten(-1, (page // 8, d, 4))
    gain = s["pool"][..., 2 * half:].view(torch.float16)
    out = []
    for x in (s["k"], s["v"]):
        x = x.double()
        norm = x.square().sum(-1).sqrt()
        unit = (x @ s["rotation"].double().T) / norm.clamp(min=1e-300)[..., None]
        out.append((_nibbles(unit, s["levels"]), norm.half()))
    (kn, kg), (vn, vg) = out
    k_codes[p, :, t] = _bytes(kn)
    gain[p, :, t], gain[p, :, page + t] = kg, vg
    # two tokens of one byte are never written by the same statement: even ones first, then odd ones
    for odd in (0, 1):
        at = (t % 2 == odd).nonzero()[:, 0]
        where = (p[at], slice(None), t[at] // 8, slice(None), t[at] % 8 // 2)
        v_bytes[where] = (v_bytes[where] & (15 if odd else 240)) | vn[at] << 4 * odd
    back = lambda nib, gains: ((_sign_magnitude(s["levels"])[nib.int()] * gains.float()[..., None]) @ s["rotation"]).to(s["k"].dtype)  # noqa: E731
    byte = v_bytes[p, :, t // 8, :, t % 8 // 2]
    read_k = torch.stack([k_codes[p, :, t] & 15, k_codes[p, :, t] >> 4], dim=-1).flatten(-2)
    read_v = (byte >> (t % 2 * 4).to(torch.uint8)[:, None, None]) & 15
    return {"k": back(read_k, gain[p, :, t]), "v": back(read_v, gain[p, :, page + t])}


def _plain_attend(s):
    c = s["case"]
    h, d, page = c["heads"], c["d"], c["page"]
    columns = -(-s["longest"] // page)
    k, v = _stored(s, s["table"][:, :columns].long().clamp(min=0))
    k, v = (x.transpose(1, 2).reshape(c["batch"], h, columns * page, d) for x in (k, v))
    seq, pos, inside = _places(s)
    q = s["q"].float()
    if c["cache"] == "code4":
        q = q @ s["rotation"].T
    full = torch.zeros(c["batch"], s["most_new"], h, c["group"], d, device=DEV)
    full[seq, inside] = q.view(-1, h, c["group"], d)
    place = torch.full((c["batch"], s["most_new"]), -1, device=DEV)
    place[seq, inside] = pos
    rows = full.permute(0, 2, 3, 1, 4).reshape(c["batch"], h, -1, d)
    scores = (rows @ k.transpose(-1, -2)).mul_(1 / math.sqrt(d)).view(c["batch"], h, c["group"], s["most_new"], -1)
    key = torch.arange(columns * page, device=DEV)
    seen = key <= place[..., None]
    if c["window"]:
        seen &= (key > place[..., None] - c["window"]) | (key < c["sinks"])
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-1e30)
    scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True)
    v = torch.where((key[None] < s["lengths"][:, None])[:, None, :, None], v, 0)
    o = (scores.view(c["batch"], h, -1, key.numel()) @ v).view(c["batch"], h, c["group"], s["most_new"], d) / torch.where(total > 0, total, 1)
    o = o.permute(0, 3, 1, 2, 4)[seq, inside].reshape(-1, h * c["group"], d)
    return (o @ s["rotation"] if c["cache"] == "code4" else o).to(s["q"].dtype)


# ---------------------------------------------------------------------------------------------------- pages

def _page_plan(case):
    lens = _sizes({**case, "new": 0, "past": case["past"]})[0]
    return lens, [-(-n // case["page"]) for n in lens]


def _columns(case):
    return -(-(case["past"] + 1 + case.get("new", 0)) // case["page"])


def _pool_pages(case):
    pages = sum(_page_plan(case)[1])
    return pages + max(4, pages // 8)


def _turn(case):
    """Parents that are forked, rows that are freed: fixed by the case."""
    r = random.Random("turn %(batch)d %(forks)d" % case)
    chosen = r.sample(range(case["batch"]), case["forks"] + case["frees"])
    return chosen[: case["forks"]], chosen[case["forks"]:]


def _compact_used(case):
    """The pages that stay in use, for `work`: pages go to sequences in an order fixed by the case."""
    _, pages = _page_plan(case)
    return _page_order(case)[sum(pages[: case["frees"]]): sum(pages)]


def _page_order(case):
    return np.random.RandomState(case["batch"] * 7 + case["page"]).permutation(_pool_pages(case))


def _prepare_pages(case, seed):
    lens, pages = _page_plan(case)
    rows, columns, count = case["batch"] + case.get("forks", 0), _columns(case), _pool_pages(case)
    order = _page_order(case)
    table = np.full((rows, columns), -1, np.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at: at + n]
        at += n
    refs = np.zeros(count, np.int32)
    refs[order[:at]] = 1
    length = np.array(lens + [0] * (rows - case["batch"]), np.int32)
    if case["op"] == "compact":  # the first conversations have ended
        for b in range(case["frees"]):
            refs[table[b, : pages[b]]] = 0
            table[b], length[b] = -1, 0
    # the whole bookkeeping in one piece, so that a pass can begin from the same state
    first = torch.from_numpy(np.concatenate([table.reshape(-1), length, refs])).to(DEV)
    now = first.clone()
    s = {"case": case, "first": first, "now": now, "table": now[: rows * columns].view(rows, columns), "lengths": now[rows * columns: rows * columns + rows],
         "refs": now[rows * columns + rows:], "pools": torch.randint(-2**31, 2**31 - 1, (case["layers"], count, case["record"] // 4), generator=_rng(seed),
                                                                     device=DEV, dtype=torch.int32)}
    if case["op"] == "turn":
        parents, freed = _turn(case)
        s["parents"] = torch.tensor(parents, dtype=torch.int32, device=DEV)
        s["children"] = torch.arange(case["batch"], rows, dtype=torch.int32, device=DEV)
        s["freed"] = torch.tensor(freed, dtype=torch.int32, device=DEV)
        s["counts"] = torch.randint(0, case["new"] + 1, (rows,), generator=_rng(seed + 1), device=DEV, dtype=torch.int32)
        s["counts"][s["freed"].long()] = 0
    return s


def _plain_turn(s):
    page, table, lengths, refs = s["case"]["page"], s["table"], s["lengths"], s["refs"]
    columns = torch.arange(table.shape[1], device=DEV)
    # freed: references fall, rows empty
    gone = table[s["freed"].long()].flatten()
    refs.index_add_(0, gone.clamp(min=0).long(), -(gone >= 0).int())
    table[s["freed"].long()] = -1
    lengths[s["freed"].long()] = 0
    # forked: full pages shared, a page that is not full copied to the lowest free one
    p, c = s["parents"].long(), s["children"].long()
    n = lengths[p]
    part = n % page != 0
    free = torch.sort(torch.where(refs == 0, torch.arange(refs.numel(), device=DEV), refs.numel())).values
    take = free[(part.cumsum(0) - 1).clamp(min=0)]
    done = ~part | (take < refs.numel())
    row = torch.where(columns[None] < (n // page)[:, None], table[p], -1)
    refs.index_add_(0, row.flatten().clamp(min=0).long(), (row.flatten() >= 0).int())
    last = (n // page).long()[:, None]
    row.scatter_(1, last.clamp(max=row.shape[1] - 1), torch.where(part, take, row.gather(1, last.clamp(max=row.shape[1] - 1))[:, 0].long()).int()[:, None])
    table[c] = row
    lengths[c] = n
    refs.index_add_(0, torch.where(done, take, 0), (part & done).int())
    source = table[p].gather(1, last.clamp(max=row.shape[1] - 1))[:, 0].long()
    s["pools"][:, take[part]] = s["pools"][:, source[part]]
    # reserved: the lowest free pages, in the order of the rows
    have, want = (lengths + page - 1) // page, (lengths + s["counts"] + page - 1) // page
    need = torch.where(want <= table.shape[1], want - have, 0)
    free = torch.sort(torch.where(refs == 0, torch.arange(refs.numel(), device=DEV), refs.numel())).values
    total = need.cumsum(0)
    fits = (want <= table.shape[1]) & ((need == 0) | (total <= (refs == 0).sum()))
    new = fits[:, None] & (columns[None] >= have[:, None]) & (columns[None] < want[:, None])
    given = free[((total - need)[:, None] + columns[None] - have[:, None]).clamp(0, refs.numel() - 1)]
    table.copy_(torch.where(new, given, table).int())
    refs.index_add_(0, torch.where(new, given, 0).flatten(), new.flatten().int())
    granted = torch.where(fits, s["counts"], 0)
    lengths += granted
    return {"state": s["now"], "done": done.int(), "granted": granted, "pools": s["pools"]}


def _plain_compact(s):
    refs, table, count = s["refs"], s["table"], s["refs"].numel()
    at = torch.arange(count, device=DEV)
    used = (refs > 0).sum()
    high, hole = (refs > 0) & (at >= used), (refs == 0) & (at < used)
    source = torch.sort(torch.where(high, at, count)).values
    target = torch.sort(torch.where(hole, at, count)).values
    moves = high.sum()
    source, target = source[:moves], target[:moves]
    new = at.clone()
    new[source] = target
    table.copy_(torch.where(table >= 0, new[table.clamp(min=0).long()], -1).int())
    refs[target] = refs[source]
    refs[source] = 0
    s["pools"][:, target] = s["pools"][:, source]
    return {"state": s["now"], "used": used.int().reshape(1), "pools": s["pools"]}


# ---------------------------------------------------------------------------------------------------- a pass

def run(s):
    op = s["case"]["op"]
    if op in ("turn", "compact"):
        s["now"].copy_(s["first"])
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "turn": _plain_turn, "compact": _plain_compact}[op](s)
    import paper_2605_17415_amd as pkg

    if op == "append":
        pkg.kv_append(s["pool"], s["k"], s["v"], s["table"], s["lengths"], starts=s["starts"], rotation=s["rotation"], levels=s["levels"])
        pkg.kv_read(s["pool"], s["table"], s["lengths"], s["k_back"], s["v_back"], starts=s["starts"], rotation=s["rotation"], levels=s["levels"])
        return {"k": s["k_back"], "v": s["v_back"]}
    if op == "attend":
        return pkg.kv_attend(s["q"], s["pool"], s["table"], s["lengths"], starts=s["starts"], max_new=s["most_new"], window=s["case"]["window"],
                             sinks=s["case"]["sinks"], rotation=s["rotation"], levels=s["levels"])
    if op == "turn":
        pkg.kv_free(s["table"], s["lengths"], s["refs"], s["freed"])
        done = pkg.kv_fork(s["pools"], s["table"], s["lengths"], s["refs"], s["parents"], s["children"], page=s["case"]["page"])
        granted = pkg.kv_reserve(s["table"], s["lengths"], s["refs"], s["counts"], page=s["case"]["page"])
        return {"state": s["now"], "done": done, "granted": granted, "pools": s["pools"]}
    used = pkg.kv_compact(s["pools"], s["table"], s["refs"])
    return {"state": s["now"], "used": used, "pools": s["pools"]}


# ---------------------------------------------------------------------------------------------------- in 64 bits

def _value(levels, nibble):
    """The level that a half byte stands for."""
    size = torch.from_numpy(levels[8:].astype(np.float64)).to(DEV)[(nibble % 8).long()]
    return torch.where(nibble >= 8, -size, size)


def _exact_append(s):
    out = {}
    for name in ("k", "v"):
        x = s[name].double()
        if s["case"]["cache"] == "code4":
            turn, norm = s["rotation"].double(), x.norm(dim=-1, keepdim=True)
            level = torch.from_numpy(s["levels"].astype(np.float64)).to(DEV)
            spun = torch.einsum("thj,ij->thi", x, turn) / norm
            code = (spun[..., None] >= (level[1:] + level[:-1]) / 2).sum(-1) if spun.numel() < 3e7 else torch.bucketize(spun, (level[1:] + level[:-1]) / 2, right=True)
            x = torch.einsum("thi,ij->thj", level[code], turn) * norm.half().double()
        out[name] = x
    return out


def _exact_attend(s):
    c, out = s["case"], []
    lens, news = _sizes(c)
    h, d, page, group, row = c["heads"], c["d"], c["page"], c["group"], 0
    for b, (n, m) in enumerate(zip(lens, news)):
        got = s["pool"][s["table"][b, : -(-n // page)].long()]
        if c["cache"] == "code4":
            half = page * d // 2
            k, v = ({0: x % 16, 1: x // 16} for x in (got[..., :half], got[..., half:2 * half]))
            k, v = (_value(s["levels"], torch.stack([x[0], x[1]], -1).flatten(-2)) for x in (k, v))
            norms = got[..., 2 * half:].contiguous().view(torch.float16).double()
            k = k.unflatten(-1, (page, d)) * norms[..., :page, None]
            v = v.unflatten(-1, (page // 8, d, 8)).permute(0, 1, 2, 4, 3).flatten(2, 3) * norms[..., page:, None]
            k, v = (x @ s["rotation"].double() for x in (k, v))
        else:
            k = got[:, :, 0].double()
            v = got[:, :, 1].double().reshape(-1, h, page // 8, d, 8).permute(0, 1, 2, 4, 3).reshape(-1, h, page, d)
        k, v = (x.permute(1, 0, 2, 3).reshape(h, -1, d)[:, :n] for x in (k, v))
        q = s["q"][row: row + m].double().view(m, h, group, d)
        row += m
        at, key = torch.arange(n - m, n, device=DEV)[:, None], torch.arange(n, device=DEV)[None]
        seen = key <= at
        if c["window"]:
            seen = seen & ((key > at - c["window"]) | (key < c["sinks"]))
        o = torch.empty(m, h, group, d, dtype=torch.float64, device=DEV)
        for i in range(h):
            for j in range(group):
                p = torch.softmax((q[:, i, j] @ k[i].T / math.sqrt(d)).masked_fill(~seen, -math.inf), dim=-1)
                o[:, i, j] = p @ v[i]
        out.append(o.view(m, h * group, d))
    return torch.cat(out)


def exact(case, seed):
    if case["op"] in ("turn", "compact"):
        return None
    s = prepare(case, seed)
    return _exact_append(s) if case["op"] == "append" else _exact_attend(s)
