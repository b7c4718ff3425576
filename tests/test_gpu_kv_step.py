"""Decoding steps as a server makes them: rows appended, digests brought up to date, pages chosen, attention over them, a token sampled; conversations
forked, ended and brought together in between; the step recorded into a graph; every call on a busy device's side stream; the example."""
import os
import sys

import numpy as np
import pytest

import kv_pick_reference as pick
import kv_reference as ref
import sample_reference

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _pkg():
    import paper_2605_17415_amd as pkg
    return pkg


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def starts_of(news):
    return ints([0] + list(np.cumsum(news)))


def rows(seed, n, heads, d=64, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(n, heads, d, generator=g).to(dtype).to(DEV) for _ in range(2)]


def check_digests(cache):
    """Every page in use has the digest that its tokens give afresh."""
    lens = cache.lengths.tolist()
    for layer in range(cache.pools.shape[0]):
        box = torch.zeros_like(cache.digests[layer])
        _pkg().kv_digest(cache.pools[layer], box, cache.table, cache.lengths, starts=starts_of(lens), **cache._codec)
        used = sorted({int(cache.table[r, c]) for r, n in enumerate(lens) for c in range(-(-n // cache.page))} - {-1})
        assert torch.equal(box[used], cache.digests[layer][used])


def step(cache, news, seed, count):
    """Returns the largest difference between attention over the chosen pages and over all of them, relative to the values."""
    starts, n = starts_of(news), sum(news)
    assert cache.reserve(ints(news)).tolist() == list(news)
    far = 0.0
    for layer in range(cache.pools.shape[0]):
        k, v = rows(seed + layer, n, cache.heads, cache.d)
        q = rows(seed + 50 + layer, n, 2 * cache.heads, cache.d)[0]
        cache.append(layer, k, v, starts)
        chosen = cache.select(layer, q, count, starts, max_new=max(news))
        some = cache.attend(layer, q, starts, max_new=max(news), pages=chosen)
        everything = cache.attend(layer, q, starts, max_new=max(news))
        far = max(far, float((some.float() - everything.float()).abs().max()))
    return far


@pytest.mark.parametrize("codes", (False, True))
def test_conversations(codes):
    cache = _pkg().KVCache(2, 2, 64, pages=70, sequences=4, tokens=400, page=16, codes=codes, device=DEV, digests=True)
    step(cache, [100, 41, 16, 0], 1, 4)
    check_digests(cache)
    assert cache.fork(ints([0, 2]), ints([3, 0])).tolist() == [1, 0]           # row 0 is not empty
    check_digests(cache)
    for n in range(20):                                                        # parent and child go different ways from a shared beginning
        step(cache, [1, n % 2, 1, 1], 100 + 10 * n, 3)
        check_digests(cache)
    cache.free(ints([0]))
    cache.compact()
    check_digests(cache)
    # as many pages as there are: the same as attention over all of them.  Both round weights and results once: 2^-8 each, of values up to 5;
    # codes: their own roundings of 2^-11 too
    assert step(cache, [33, 2, 0, 7], 900, 25) <= 4 * 2.0 ** -8 * 5
    check_digests(cache)
    cache.trim(32, 16)
    step(cache, [1, 1, 1, 1], 950, 4)
    assert cache.lengths.tolist() == [34, 54, 37, 128]


def test_pages_without_digests_are_refused():
    cache = _pkg().KVCache(1, 1, 64, pages=4, sequences=1, tokens=40, page=16, device=DEV)
    q = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        cache.select(0, q, 2)
    with pytest.raises(ValueError):
        cache.attend(0, q, window=5, pages=torch.zeros(1, 1, 1, dtype=torch.int32, device=DEV))


@pytest.mark.parametrize("codes", (False, True))
def test_a_refused_reservation_leaves_digests_alone(codes):
    cache = _pkg().KVCache(1, 1, 64, pages=3, sequences=2, tokens=64, page=16, codes=codes, device=DEV, digests=True)
    step(cache, [20, 10], 3, 2)
    before = cache.digests.clone()
    news = [1, 30]
    assert cache.reserve(ints(news)).tolist() == [1, 0]
    k, v = rows(9, 31, 1)
    cache.append(0, k, v, starts_of(news))
    check_digests(cache)
    pages = {int(cache.table[1, 0])}
    assert all(torch.equal(cache.digests[0, p], before[0, p]) for p in pages)


@pytest.mark.parametrize("codes", (False, True))
def test_a_recorded_step(codes):
    """Reserve, append, choose, attend and sample recorded once and replayed, with eager steps of the same state between the replays."""
    pkg, batch, heads, group = _pkg(), 3, 2, 4
    cache = pkg.KVCache(1, heads, 64, pages=60, sequences=batch, tokens=300, page=16, codes=codes, device=DEV, digests=True)
    step(cache, [200, 50, 7], 1, 4)
    k, v = rows(5, batch, heads)
    q = rows(6, batch, heads * group)[0]
    out_of = (torch.randn(heads * group * 64, 5000, generator=torch.Generator().manual_seed(1)) / 8).to(DEV)
    one, u = ints([1] * batch), torch.zeros(batch, device=DEV)
    lse, logs = torch.zeros(batch, heads * group, device=DEV), torch.zeros(batch, device=DEV)
    settings = {"temperature": torch.tensor([0.7, 1.0, 0.0], device=DEV), "top_p": torch.tensor([0.9, 1.0, 0.5], device=DEV), "top_k": ints([0, 30, 4])}

    def go():
        cache.reserve(one)
        cache.append(0, k, v)
        chosen = cache.select(0, q, 4)
        out = cache.attend(0, q, pages=chosen, lse=lse)
        logits = out.float().flatten(1) @ out_of
        return chosen, out, logits, pkg.sample_tokens(logits, u, logprobs=logs, **settings)

    parts = (cache.table, cache.lengths, cache.refs, cache.pools, cache.digests, cache._asked, cache._granted)
    first = [x.clone() for x in parts]
    go()
    for x, y in zip(parts, first):
        x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = go()
    for n in range(20):                                     # row 2 begins a page in between
        for x, seed in ((k, 10 + n), (v, 40 + n)):
            x.copy_(rows(seed, batch, heads)[0])
        q.copy_(rows(70 + n, batch, heads * group)[0])
        u.copy_(torch.rand(batch, generator=torch.Generator().manual_seed(n)))
        before = [x.clone() for x in parts]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (*recorded, lse, logs, *parts)]
        for x, y in zip(parts, before):
            x.copy_(y)
        eager = (*go(), lse, logs, *parts)
        for x, y in zip(got[:2] + got[4:5] + got[6:], eager[:2] + eager[4:5] + eager[6:]):
            assert torch.equal(x.float().nan_to_num(), y.float().nan_to_num())
        # the library's product may round otherwise in a graph: the tokens are those of the logits that it gave
        for r in range(batch):
            token, log = sample_reference.sample(got[2][r].double().cpu().numpy(), float(u[r]), float(settings["temperature"][r]), int(settings["top_k"][r]),
                                                 float(settings["top_p"][r]))
            assert int(got[3][r]) == token and abs(float(got[5][r]) - log) <= 2.0 ** -22 * abs(log) + 1e-9
    assert cache.lengths.tolist() == [220, 70, 27]


def busy():
    """Some milliseconds of work on the current stream."""
    x = torch.ones(4096, 4096, device=DEV, dtype=torch.bfloat16)
    for _ in range(20):
        x = x @ x
    return x


@pytest.mark.parametrize("form,kind", [("bf16", "bf16"), ("code4", "f16")])
@pytest.mark.parametrize("news", ([1, 1], [70, 9]))
def test_on_a_side_stream(form, kind, news):
    pkg = _pkg()
    lens = [2500, 900]
    c = ref.Cache(31, form, 2, 64, 16, lens)
    t, codec = c.device()
    q = (torch.randn(sum(news), 4, 64, generator=torch.Generator().manual_seed(3))).to(ref.TYPES[kind]).to(DEV)
    box = [torch.zeros(c.pages, 2, 2, 64, dtype=torch.float16 if form == "code4" else ref.TYPES[form], device=DEV) for _ in range(2)]
    logits, u, side = torch.randn(5, 40_000, device=DEV), torch.rand(5, device=DEV), torch.cuda.Stream()
    every, starts = starts_of(lens), starts_of(news)
    how = {"starts": starts, "max_new": max(news)}

    def go(box, **on):
        pkg.kv_digest(t["pool"], box, t["table"], t["lengths"], starts=every, **codec, **on)
        scores = pkg.kv_score(q, box, t["pool"], t["table"], t["lengths"], **how, **codec, **on)
        chosen = pkg.kv_select(scores, t["lengths"], 16, 7, starts=starts, **on)
        return scores, chosen, pkg.kv_attend_pages(q, t["pool"], t["table"], t["lengths"], chosen, **how, **codec, **on), pkg.sample_tokens(logits, u, top_p=0.9, **on)

    torch.cuda.synchronize()
    for _ in range(2):                                      # the second time memory is there to be handed out again
        keep = busy()
        here = go(box[0])
        there = go(box[1], stream=side)
        torch.cuda.synchronize()
        del keep
        for x, y in zip(here, there):
            assert torch.equal(x, y)
        pick.check_attention(c, q.cpu(), there[2], news, there[1].cpu().numpy())


@pytest.mark.parametrize("codes", (False, True))
def test_generation(codes):
    """The example with pages of each token's own choice and sampled tokens."""
    from generate import generate
    plain, _, used = generate(codes=codes, steps=12, pages=3)
    assert [len(t) for t in plain] == [49, 12, 102, 49] and used > 0
    whole, off, _ = generate(codes=codes, steps=12, pages=12, check=True)
    assert off < (0.3 if codes else 0.06)                   # every page is among the chosen ones: as without a choice
    a, _, _ = generate(codes=codes, steps=12, pages=3, temperature=0.9, top_k=50, top_p=0.95, min_p=0.01)
    b, _, _ = generate(codes=codes, steps=12, pages=3, temperature=0.9, top_k=50, top_p=0.95, min_p=0.01)
    assert a == b and all(0 <= t < 256 for text in a for t in text) and a[0][:37] == plain[0][:37]
