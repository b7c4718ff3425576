"""Text generation with the paged key-value cache: a small random-weight transformer answers several prompts of unequal length,
one prompt is forked into two answers, tokens are made one at a time, ended conversations give their pages back and the pool is
brought together.

    python examples/generate.py [--codes] [--window 64 --sinks 4] [--steps 24]

With --check every step's logits are compared with a full recomputation in float32 that keeps no cache.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2605_17415_amd as ivftq  # noqa: E402


class Model:
    """Embedding, `layers` times (attention with grouped heads, two-layer perceptron) on normalised rows, logits."""

    def __init__(self, vocabulary=256, layers=2, width=256, heads=8, kv_heads=2, d=64, seed=0, device="cuda", dtype=torch.bfloat16):
        g = torch.Generator().manual_seed(seed)
        make = lambda *shape: (torch.randn(*shape, generator=g) / shape[0] ** 0.5).to(device, dtype)  # noqa: E731
        self.heads, self.kv_heads, self.d, self.layers = heads, kv_heads, d, layers
        self.embed = make(vocabulary, width) * vocabulary ** 0.5
        self.place = make(4096, width) * 4096 ** 0.5 * 0.5
        self.blocks = [{"qkv": make(width, (heads + 2 * kv_heads) * d), "out": make(heads * d, width), "up": make(width, 4 * width), "down": make(4 * width, width)}
                       for _ in range(layers)]

    def __call__(self, tokens, positions, attention):
        """Logits of rows of tokens at positions; attention(layer, q, k, v) sees what the rows see."""
        norm = lambda x: x * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6).to(x.dtype)  # noqa: E731
        x = self.embed[tokens] + self.place[positions]
        for i, b in enumerate(self.blocks):
            qkv = (norm(x) @ b["qkv"]).view(x.shape[0], -1, self.d)
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
            x = x + attention(i, q, k, v).reshape(x.shape[0], -1) @ b["out"]
            x = x + torch.relu(norm(x) @ b["up"]) @ b["down"]
        return norm(x).float() @ self.embed.float().T / x.shape[1] ** 0.5


def recompute(model, tokens, window, sinks):
    """The last row's logits of one sequence, in float32 and without a cache."""
    wide = Model.__new__(Model)
    wide.__dict__.update(model.__dict__, embed=model.embed.float(), place=model.place.float(), blocks=[{k: v.float() for k, v in b.items()} for b in model.blocks])
    n = len(tokens)
    at = torch.arange(n, device=model.embed.device)
    seen = at[None] <= at[:, None]
    if window:
        seen &= (at[None] > at[:, None] - window) | (at[None] < sinks)

    def attention(_, q, k, v):
        q, k, v = q.float(), k.float().repeat_interleave(model.heads // model.kv_heads, 1), v.float().repeat_interleave(model.heads // model.kv_heads, 1)
        s = (q.transpose(0, 1) @ k.permute(1, 2, 0).contiguous()) / model.d ** 0.5
        return (torch.softmax(s.masked_fill(~seen, -torch.inf), -1) @ v.transpose(0, 1).contiguous()).transpose(0, 1)

    return wide(torch.tensor(tokens, device=at.device), at, attention)[-1]


def generate(codes=False, window=0, sinks=0, steps=24, check=False, page=16, prompts=(37, 5, 90), seed=0):
    """Returns (token lists, largest difference of logits from the recomputation relative to their spread, pages left in use)."""
    device = torch.device("cuda", torch.cuda.current_device())
    model = Model(seed=seed, device=device)
    rows = len(prompts) + 1                                                       # one more for the fork
    cache = ivftq.KVCache(model.layers, model.kv_heads, model.d, pages=rows * (max(prompts) + steps + page) // page + rows, sequences=rows,
                          tokens=max(prompts) + steps + 1, page=page, codes=codes, device=device)
    g = torch.Generator().manual_seed(seed + 1)
    texts = [torch.randint(0, 256, (n,), generator=g).tolist() for n in prompts] + [[]]
    worst = 0.0

    def step(new):
        """new[r]: tokens of row r that the cache has not seen; logits of each row's last one."""
        counts = torch.tensor([len(t) for t in new], dtype=torch.int32, device=device)
        granted = cache.reserve(counts)
        if not torch.equal(granted, counts):
            raise RuntimeError("the cache is full")
        starts = torch.cat([counts.new_zeros(1), counts.cumsum(0, dtype=torch.int32)])
        flat = torch.tensor([t for row in new for t in row], device=device)
        positions = torch.cat([torch.arange(len(texts[r]) - len(t), len(texts[r]), device=device) for r, t in enumerate(new)])

        def attention(layer, q, k, v):
            cache.append(layer, k, v, starts)
            return cache.attend(layer, q, starts, max_new=max(map(len, new)), window=window, sinks=sinks)

        return model(flat, positions, attention)[(starts[1:] - 1).long().clamp(min=0)]

    logits = step(texts)
    cache.fork(torch.tensor([0], dtype=torch.int32, device=device), torch.tensor([rows - 1], dtype=torch.int32, device=device))
    texts[-1] = list(texts[0])
    logits[-1] = logits[0]
    live = list(range(rows))
    for n in range(steps):
        best = logits.topk(2).indices.tolist()
        new = [[] for _ in range(rows)]
        for r in live:
            new[r] = [best[r][1] if n == 0 and r == rows - 1 else best[r][0]]      # the fork begins with the second best token
            texts[r] += new[r]
        logits = step(new)
        if check:
            for r in live:
                exact = recompute(model, texts[r], window, sinks)
                worst = max(worst, float((logits[r] - exact).norm() / exact.norm()))
        if window:
            cache.trim(window, sinks)
        if n == steps // 2:                                                       # the second conversation ends
            live.remove(1)
            cache.free(torch.tensor([1], dtype=torch.int32, device=device))
            cache.compact()
    return texts, worst, int(cache.refs.gt(0).sum())


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--codes", action="store_true", help="keep keys and values in 4-bit codes")
    parser.add_argument("--window", type=int, default=0)
    parser.add_argument("--sinks", type=int, default=0)
    parser.add_argument("--steps", type=int, default=24)
    parser.add_argument("--check", action="store_true")
    a = parser.parse_args()
    got, off, used = generate(a.codes, a.window, a.sinks, a.steps, a.check)
    for r, text in enumerate(got):
        print(f"row {r}: {len(text)} tokens, the last {text[-8:]}")
    print(f"{used} pages in use" + (f", logits {off:.3g} from the recomputation" if a.check else ""))
