"""Plain float64 numpy oracle of sampling (pctree_sample in include/pctree.h).

Test infrastructure only; nothing in the product path imports it.
"""
from __future__ import annotations

import math

import numpy as np


def sample_row(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob, margin) of one row.  margin: the smallest relative distance of
    a decision (a kept set's border, the draw) from its border, of the two that sums
    decide (inf: neither did)."""
    x = np.asarray(logits, np.float64).copy()
    x[np.isnan(x)] = -np.inf
    best = x.max()
    if best == -np.inf:
        return -1, -math.inf, math.inf
    if not temperature > 0:
        return int(np.argmax(x)), 0.0, math.inf
    with np.errstate(invalid="ignore", over="ignore"):
        z = np.where(x == best, 0.0, np.where(x == -np.inf, -np.inf, (x - best) / np.float64(temperature)))
        w = np.where(z >= -700.0, np.exp(np.minimum(z, 0.0)), 0.0)
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[x[order] > -np.inf]
    margin = math.inf
    n = len(order)
    if min_p > 0:
        n = max(int((w[order] >= min(min_p, 1.0)).sum()), 1)
    if top_k > 0:
        n = min(n, top_k)
    if top_p < 1:
        cum = np.cumsum(w[order[:n]])
        before = np.concatenate([[0.0], cum[:-1]])
        limit = top_p * cum[-1]
        m = max(int((before < limit).sum()), 1)
        if limit > 0:
            margin = min(margin, float(np.abs(cum[:m + 1] - limit).min() / cum[-1]))
        n = m
    kept = np.sort(order[:n])
    cum = np.cumsum(w[kept])
    total = cum[-1]
    u = 0.0 if not u > 0 else float(u)
    past = np.nonzero(cum > u * total)[0]
    j = int(past[0]) if len(past) else int(np.nonzero(w[kept] > 0)[0][-1])
    if 0 < u < 1:
        margin = min(margin, float(np.abs(cum - u * total).min() / total))
    zt = z[kept[j]]
    return int(kept[j]), float(zt - math.log(total)), margin


def sample(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None):
    """(tokens, logprobs, margins) of every row."""
    def at(p, t, off):
        return off if p is None else p[t]
    rows = [sample_row(logits[t], uniform[t], at(temperature, t, 1.0), at(top_k, t, 0), at(top_p, t, 1.0),
                       at(min_p, t, 0.0)) for t in range(len(uniform))]
    return tuple(np.array(c) for c in zip(*rows))
