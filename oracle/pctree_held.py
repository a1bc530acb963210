"""Plain float64 numpy oracle of a paged cache in 8 bits (include/pctree.h): scales, held
values, appended rows, compaction.  Attention is that of ``pctree_paged`` over the values.

Test infrastructure only; nothing in the product path imports it.
"""
from __future__ import annotations

import math

import numpy as np

from . import pctree_paged as PO

LEAST, MOST = 16, 246


def numbers():
    """The value of each e4m3 byte."""
    out = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = math.nan if b & 127 == 127 else math.ldexp(8 + m, e - 10) if e else math.ldexp(m, -9)
        out[b] = -v if b & 128 else v
    return out


NUMBERS = numbers()


def scale_byte(largest):
    """The smallest scale with which ``largest`` is at most 448 times it."""
    for s in range(LEAST, MOST):
        if largest <= 448.0 * 2.0 ** (s - 127):
            return s
    return MOST


def hold(x, s):
    """The bytes of values ``x`` under scale ``s``: the nearest numbers, ties to the even byte."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore"):
        z = np.abs(x) * 2.0 ** (127 - s)
    pos = NUMBERS[:127]
    i = np.clip(np.searchsorted(pos, np.nan_to_num(z, nan=0.0, posinf=0.0)), 1, 126)
    lo, hi = pos[i - 1], pos[i]
    mid = (lo + hi) / 2
    b = np.where((z > mid) | ((z == mid) & (i % 2 == 0)), i, i - 1)
    b = np.where(z > 464.0, 127, b)
    b = np.where(np.isfinite(z), b, 127)
    return (b | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def values(pages, scale):
    """What pages [..., slots, D] hold under scales [..., blocks], both bytes."""
    G = pages.shape[-2] // scale.shape[-1]
    s = np.clip(scale.astype(np.int64), LEAST, MOST) - 127
    return NUMBERS[pages] * np.repeat(2.0 ** s, G, -1)[..., None]


def rescale(b, was, now):
    """Bytes under the scale ``was`` held again under ``now``."""
    return b if was == now else np.where(b & 127 == 127, b, hold(NUMBERS[b] * 2.0 ** (was - 127), now))


def largest(x):
    a = np.abs(np.asarray(x, np.float64))
    a = a[np.isfinite(a)]
    return float(a.max()) if a.size else 0.0


def touched_blocks(batch, P, pages, G):
    """[(request, page, first slot of the block in the page, slots held before, rows)] of every
    block that takes new rows; rows: [(row, offset in the block)]."""
    blocks = {}
    for r, t, i, prefix, _ in PO.live_rows(batch, P):
        at = PO.place(batch, r, prefix + i, P, pages)
        if at is None:
            continue
        page, off = at
        first = off // G * G
        old = max(min(prefix - (prefix + i - (off - first)), G), 0)
        blocks.setdefault((r, page, first), (old, []))[1].append((t, off - first))
    return [(r, p, f, old, rows) for (r, p, f), (old, rows) in blocks.items()]


def compact(pool, scale, table, prefix, accept_node, accept_len, budget):
    """(pool [G][pages][heads][P][D], scale [G][pages][heads][P / block]) bytes after compaction."""
    pool, scale = pool.copy(), scale.copy()
    old, olds = pool.copy(), scale.copy()
    groups, pages, heads, P, _ = pool.shape
    G = P // scale.shape[3]
    b = {"page_table": table}
    for r in range(len(prefix)):
        a, W, p = int(accept_len[r]), accept_node.shape[1], int(prefix[r])
        if not 0 <= a < W or p < 0:
            continue
        nodes = [int(x) for x in accept_node[r, :a + 1]]
        if any(x < 0 or x >= budget for x in nodes) or any(x >= y for x, y in zip(nodes, nodes[1:])):
            continue
        if any(p + x >= table.shape[1] * P for x in nodes) or nodes == list(range(a + 1)):
            continue
        src = [PO.place(b, r, p + x, P, pages) for x in nodes]
        dst = [PO.place(b, r, p + m, P, pages) for m in range(a + 1)]
        if any(x is None for x in src + dst):
            continue
        for g in range(groups):
            for h in range(heads):
                by = lambda at: int(np.clip(olds[g, at[0], h, at[1] // G], LEAST, MOST))  # noqa: E731
                for first in range(p // G * G, p + a + 1, G):
                    mine = [m for m in range(a + 1) if first <= p + m < first + G]
                    now = max(by(src[m]) for m in mine)
                    page, off = PO.place(b, r, first, P, pages)
                    if first < p:
                        was = by((page, off))
                        now = max(now, was)
                        for s in range(first, p):
                            o = off + s - first
                            pool[g, page, h, o] = rescale(old[g, page, h, o], was, now)
                    for m in mine:
                        (sp, so), (dp, do) = src[m], dst[m]
                        pool[g, dp, h, do] = rescale(old[g, sp, h, so], by(src[m]), now)
                    scale[g, page, h, off // G] = now
    return pool, scale
