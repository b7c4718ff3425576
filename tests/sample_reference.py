"""Sampling from its definition: weights in float64 as whole multiples of 2^-42, ranks by sorting, sums in whole numbers."""
import math

import numpy as np


def weights(x, temperature):
    """The row's weights in float64; x without what is no number."""
    top = x.max()
    if top == np.inf:
        return (x == np.inf).astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.exp((x - top) / np.float64(temperature))
    w[x == -np.inf] = 0.0
    w[x == top] = 1.0
    return w


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log of its probability) of one row."""
    x = np.asarray(x, np.float64).copy()
    x[np.isnan(x)] = -np.inf
    n, f = len(x), np.float64
    if x.max() == -np.inf:
        return -1, -math.inf
    order = np.argsort(-x, kind="stable")
    if not temperature > 0:
        return int(order[0]), 0.0
    w = weights(x, temperature)
    whole = np.rint(w * 2.0 ** 42).astype(np.int64)
    if 0 < top_k < n:
        order = order[:top_k]
    if top_p < 1:
        mass = whole[order]
        before = np.cumsum(mass) - mass
        kept = before.astype(f) < f(max(np.float32(top_p), np.float32(0))) * f(mass.sum())
        kept[0] = True
        order = order[kept]
    order = np.sort(order[w[order] >= min(f(max(np.float32(min_p), np.float32(0))), 1.0)])
    upto = np.cumsum(whole[order])
    total = int(upto[-1])
    u = np.float32(u)
    target = total - 1 if u >= 1 else min(int(f(u) * f(total)), total - 1) if u > 0 else 0
    at = int(np.searchsorted(upto, target, side="right"))
    return int(order[at]), math.log(w[order[at]] / (total / 2.0 ** 42))
