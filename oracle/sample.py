"""Oracle of the token drawn from logits: temperature, top-k, top-p and min-p from
a given random number.

TEST INFRASTRUCTURE ONLY, like the rest of this package: plain numpy in fp64,
sharing no code with the GPU library.
"""
from __future__ import annotations

import numpy as np


def kept(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(tokens in descending order of their logits, their weights, how many are
    kept), or (the arg max, [1], 1)."""
    l = np.asarray(logits, np.float64)
    l = np.where(np.isnan(l), -np.inf, l)
    order = np.lexsort((np.arange(len(l)), -l))
    top = l[order[0]]
    if not temperature > 0 or top == -np.inf:
        return np.array([int(np.argmax(l))]), np.ones(1), 1
    if top == np.inf:
        w = (l[order] == np.inf).astype(np.float64)
    else:
        w = np.exp((l[order] - top) / np.float64(temperature))
        w = np.where(l[order] == -np.inf, 0.0, w)
    n = len(w)
    if 0 < top_k < n:
        n = top_k
    m = n
    if top_p < 1:
        c = np.cumsum(w[:n])
        m = min(n, int(np.sum(c < top_p * c[-1])) + 1)
    if min_p > 0:
        m = min(m, int(np.sum(w >= min(min_p, 1.0))))
    return order, w, m


def draw(logits, u, **settings):
    """(token, its share of the kept weight, distance of u's mass from the nearest border of the token's)."""
    order, w, n = kept(logits, **settings)
    u = min(max(0.0 if np.isnan(u) else float(u), 0.0), 1.0 - 2.0 ** -24)
    c = np.cumsum(w[:n])
    j = int(np.sum(c <= u * c[-1]))
    share = w[j] / c[-1]
    near = min(abs(c[j] - u * c[-1]), abs(c[j] - w[j] - u * c[-1]) if j else np.inf) / c[-1]
    return int(order[j]), share, near
