"""Plain float64 numpy oracles of the verification step over a paged cache
(include/pctree.h): appended rows, attention of new rows over pages, compaction.

Test infrastructure only; nothing in the product path imports it.
"""
from __future__ import annotations

import numpy as np


def live_rows(batch, page_size, budget=None):
    """(request, row, i, prefix, count) of every row that a request has, with the
    clamping of the interface.  ``batch``: dict of row_start, row_count, prefix_len
    [R], page_table [R][W], rows, max_rows."""
    cap = batch["page_table"].shape[1] * page_size
    out = []
    for r in range(len(batch["row_start"])):
        start = int(batch["row_start"][r])
        if not 0 <= start < batch["rows"]:
            continue
        n = min(max(int(batch["row_count"][r]), 0), batch["max_rows"], batch["rows"] - start)
        if budget is not None:
            n = min(n, budget)
        prefix = min(max(int(batch["prefix_len"][r]), 0), cap)
        out += [(r, start + i, i, prefix, n) for i in range(n)]
    return out


def place(batch, r, slot, page_size, pages):
    """(page, offset) of a request's slot, or None if it does not exist."""
    table = batch["page_table"][r]
    if slot >= len(table) * page_size:
        return None
    p = int(table[slot // page_size])
    return (p, slot % page_size) if 0 <= p < pages else None


def norm_rotate(x, weight, eps, cs, interleaved):
    """One head vector: root-mean-square norm (weight None: none) and rotation by the
    table row ``cs`` (None: none).  Returns the result and, per element, the sum of
    the magnitudes that were added for it."""
    y = np.asarray(x, np.float64)
    if weight is not None:
        y = y / np.sqrt(np.mean(y * y) + eps) * np.asarray(weight, np.float64)
    mag = np.abs(y)
    if cs is not None:
        half = len(cs) // 2
        c, s = np.asarray(cs[:half], np.float64), np.asarray(cs[half:], np.float64)
        i = np.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        z, mag = y.copy(), mag.copy()
        z[a], z[b] = y[a] * c - y[b] * s, y[b] * c + y[a] * s
        mag[a] = mag[b] = np.abs(y[a]) + np.abs(y[b])
        y = z
    return y, mag


def append(batch, k_cache, v_cache, q, k, v, q_norm, k_norm, eps, rope, interleaved, position):
    """New contents of (q_out, k_cache, v_cache) as float64 and the magnitudes of
    norm_rotate for q and k: dicts {row or (page, offset): [heads][D]}."""
    pages, _, P, _ = k_cache.shape
    qo, ko, vo = {}, {}, {}
    for r, t, i, prefix, _ in live_rows(batch, P):
        slot = prefix + i
        cs = None
        if rope is not None:
            pos = slot if position is None else int(position[t])
            cs = rope[min(max(pos, 0), len(rope) - 1)]
        if q is not None:
            qo[t] = [norm_rotate(h, q_norm, eps, cs, interleaved) for h in q[t]]
        at = place(batch, r, slot, P, pages)
        if at is not None:
            ko[at] = [norm_rotate(h, k_norm, eps, cs, interleaved) for h in k[t]]
            vo[at] = v[t]
    return qo, ko, vo


def attention(batch, q, k_cache, v_cache, scale, mask=None, budget=None):
    """{row: (out [Hq][D], sum of weight * |value| [Hq][D])} in float64.  A value
    counts only for the rows that admit its slot."""
    pages, Hkv, P, D = k_cache.shape
    Hq = q.shape[1]
    out = {}
    cap = batch["page_table"].shape[1] * P
    for r, t, i, prefix, n in live_rows(batch, P, budget):
        end = min(prefix + n, cap)
        slots = range(min(prefix, end)) if mask is not None else range(min(prefix + i + 1, end))
        slots = list(slots)
        if mask is not None:
            words = mask[r, i].astype(np.uint32)
            slots += [prefix + j for j in range(n)
                      if prefix + j < end and (int(words[j // 32]) >> (j % 32)) & 1]
        at = [a for a in (place(batch, r, s, P, pages) for s in slots) if a is not None]
        o, mag = np.zeros((Hq, D)), np.zeros((Hq, D))
        if at:
            pg, off = np.array(at).T
            for h in range(Hq):
                kk = k_cache[pg, h // (Hq // Hkv), off].astype(np.float64)
                vv = v_cache[pg, h // (Hq // Hkv), off].astype(np.float64)
                z = kk @ q[t, h].astype(np.float64) * scale
                w = np.exp(z - z.max())
                w /= w.sum()
                with np.errstate(invalid="ignore"):
                    o[h], mag[h] = w @ vv, w @ np.abs(vv)
        out[t] = (o, mag)
    return out


def compact(pool, table, prefix, accept_node, accept_len, budget):
    """The pool [G][pages][heads][P][...] after compaction (a copy)."""
    out = pool.copy()
    G, pages, _, P = pool.shape[:4]
    b = {"page_table": table}
    for r in range(len(prefix)):
        a, W = int(accept_len[r]), accept_node.shape[1]
        if not 0 <= a < W or prefix[r] < 0:
            continue
        nodes = [int(x) for x in accept_node[r, :a + 1]]
        if any(x < 0 or x >= budget for x in nodes) or any(x >= y for x, y in zip(nodes, nodes[1:])):
            continue
        cap = table.shape[1] * P
        if any(int(prefix[r]) + x >= cap for x in nodes):
            continue
        moves = [(place(b, r, int(prefix[r]) + x, P, pages), place(b, r, int(prefix[r]) + m, P, pages))
                 for m, x in enumerate(nodes)]
        if any(s is None or d is None for s, d in moves):
            continue
        for (sp, so), (dp, do) in moves:
            out[:, dp, :, do] = pool[:, sp, :, so]
    return out
