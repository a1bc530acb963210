"""Plain float64 numpy oracles of the norm before a projection and of what is done to logits
before a token is drawn (include/pctree.h).

Test infrastructure only; nothing in the product path imports it.
"""
from __future__ import annotations

import numpy as np


def rms_norm(x, weight, residual, eps):
    """(v, y): the sum and its norm."""
    v = np.asarray(x, np.float64) + (0.0 if residual is None else residual)
    y = v / np.sqrt(np.mean(v * v, 1, keepdims=True) + eps)
    return v, y if weight is None else y * weight


def group_scales(y, group):
    """max |y| / 448 of each group, finite elements only."""
    H = y.shape[1]
    a = np.where(np.isfinite(y), np.abs(y), 0.0)
    return np.stack([a[:, i:i + group].max(1) for i in range(0, H, group)], 1) / 448.0


def _at(p, r, off):
    return off if p is None else p[r]


def adjust(logits, row_start, row_count, max_rows, *, history=None, history_start=None, history_count=None,
           prompt_count=None, repetition=None, frequency=None, presence=None, bias_token=None, bias_value=None,
           bias_start=None, bias_count=None, token=None, mask=None, allowed=None, allowed_row=None):
    """(logits after, magnitude of what was added for each, which were concerned)."""
    x = np.array(logits, np.float64)
    T, V = x.shape
    mag, hit = np.abs(x), np.zeros(x.shape, bool)
    for r in range(len(row_start)):
        start = int(row_start[r])
        if not 0 <= start < T:
            continue
        n = min(max(int(row_count[r]), 0), max_rows, T - start)
        if token is not None:
            n = min(n, token.shape[1])
        said, prompt = np.zeros(0, np.int64), 0
        if history is not None:
            h0 = min(max(int(history_start[r]), 0), len(history))
            hn = min(max(int(history_count[r]), 0), len(history) - h0)
            prompt = min(max(int(_at(prompt_count, r, 0)), 0), hn)
            said = history[h0:h0 + hn].astype(np.int64)
        rep, freq, pres = (float(_at(p, r, off)) for p, off in ((repetition, 1.0), (frequency, 0.0), (presence, 0.0)))
        rep = rep if np.isfinite(rep) and rep > 0 else 1.0
        freq, pres = (f if np.isfinite(f) else 0.0 for f in (freq, pres))
        bias = {}
        if bias_token is not None:
            b0 = min(max(int(bias_start[r]), 0), len(bias_token))
            bn = min(max(int(bias_count[r]), 0), len(bias_token) - b0)
            bias = {int(t): float(v) for t, v in zip(bias_token[b0:b0 + bn], bias_value[b0:b0 + bn]) if 0 <= t < V}
        for i in range(n):
            t = start + i
            made = list(said[prompt:])
            if token is not None:
                made += [int(token[r, j]) for j in range(n) if int(mask[r, i, j // 32]) >> (j % 32) & 1]
            made = np.array([m for m in made if 0 <= m < V], np.int64)
            count = np.bincount(made, minlength=V)
            seen = count > 0
            first = said[:prompt]
            seen[first[(first >= 0) & (first < V)]] = True
            y = x[t]
            with np.errstate(invalid="ignore", over="ignore"):
                y = np.where(seen, np.where(y > 0, y / rep, y * rep), y)
                mag[t] = np.where(seen, np.abs(y), mag[t])
                y = np.where(count > 0, y - freq * count - pres, y)
                mag[t] += np.where(count > 0, abs(freq) * count + abs(pres), 0.0)
            hit[t] |= seen if (rep, freq, pres) != (1.0, 0.0, 0.0) else False
            for k, v in bias.items():
                y[k] += v
                mag[t, k] += abs(v)
                hit[t, k] = True
            if allowed is not None:
                m = t if allowed_row is None else int(allowed_row[t])
                if 0 <= m < len(allowed):
                    bits = (allowed[m].view(np.uint32)[:, None] >> np.arange(32, dtype=np.uint32)) & 1
                    no = bits.reshape(-1)[:V] == 0
                    y[no] = -np.inf
                    hit[t] |= no
            x[t] = y
    return x, mag, hit
