"""Oracle of the attention half of a decoder step and of sampling -- TEST INFRASTRUCTURE ONLY.

Plain numpy in 64 bits, one loop per token, page and head, written from the definitions in include/moe.h; it shares nothing with
the library's kernels.  ``oracle/quant_e4m3.py`` holds the number format.

    append   rotated queries, and a cache (dict of k, v bytes and k_scale, v_scale) as the call leaves it
    attend   outputs, logarithms of the denominators, and for each output sum_p softmax_p |value_p|, which error bounds are
             relative to
    sample   the token and its log-probability for a row of logits
"""
from __future__ import annotations

import math

import numpy as np

from oracle import quant_e4m3 as e4m3

VALUES = e4m3.code_values()


def needed_scale(largest: float) -> float:
    """The smallest power of two, at least 2^-126, with largest <= 448 times it."""
    n = -126
    while largest > 448.0 * 2.0 ** n:
        n += 1
    return 2.0 ** n


def rotate(x, pos, inv_freq, interleaved):
    """x [heads, head_dim] of one token, in 64 bits."""
    y = np.array(x, dtype=np.float64)
    half = len(inv_freq)
    for j, f in enumerate(inv_freq):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        c, s = math.cos(pos * f), math.sin(pos * f)
        y[:, a], y[:, b] = x[:, a] * c - x[:, b] * s, x[:, b] * c + x[:, a] * s
    return y


def append(cache, q, k, v, inv_freq, interleaved, q_offsets, kv_len, page_table, page_size, max_q=None):
    """max_q: a sequence's further new tokens are left out (their rows of the result are the queries as they came)."""
    q_out = None if q is None else np.array(q, dtype=np.float64)
    num_pages = cache["k"].shape[0]
    for b, kv in enumerate(kv_len):
        lo, hi = q_offsets[b], q_offsets[b + 1]
        begin = kv - (hi - lo)
        n = hi - lo if max_q is None else min(hi - lo, max_q)
        end = min(kv, begin + n)
        if q is not None:
            for t in range(lo, lo + n):
                q_out[t] = rotate(q[t], begin + t - lo, inv_freq, interleaved)
        first = max(begin, 0)
        for slot in range(first // page_size, -(-end // page_size) if n > 0 else 0):
            page = page_table[b][slot]
            if not 0 <= page < num_pages:
                continue
            rows = range(max(first, slot * page_size), min(end, (slot + 1) * page_size))
            if not len(rows):
                continue
            r0 = rows[0] - slot * page_size
            new = {"k": [rotate(k[lo + p - begin], p, inv_freq, interleaved).astype(np.float32).astype(np.float64) for p in rows],
                   "v": [np.array(v[lo + p - begin], dtype=np.float64) for p in rows]}
            for name in "kv":
                x = np.stack(new[name])                                     # [rows, heads, dim]
                for h in range(x.shape[1]):
                    scale = needed_scale(float(np.abs(x[:, h]).max()))
                    if r0:
                        old = float(cache[name + "_scale"][page, h])
                        scale = max(scale, old)
                        if scale > old:
                            cache[name][page, h, :r0] = e4m3.nearest_code(VALUES[cache[name][page, h, :r0]] * (old / scale))
                    cache[name + "_scale"][page, h] = scale
                    cache[name][page, h, r0:r0 + len(rows)] = e4m3.nearest_code(x[:, h] / scale)
    return q_out


def attend(cache, q, q_offsets, kv_len, page_table, page_size, scale, causal=True, window=0, max_q=None, max_kv=None):
    """max_q, max_kv: a sequence's further new tokens (rows of zeros here), and its further keys, are left out."""
    T, heads, dim = q.shape
    num_pages, kv_heads = cache["k"].shape[:2]
    out, absolute, lse = np.zeros((T, heads, dim)), np.zeros((T, heads, dim)), np.full((T, heads), -np.inf)
    spread = np.zeros((T, heads))                                          # largest sum of |q k| of a row, times scale
    for b, length in enumerate(kv_len):
        lo, hi = q_offsets[b], q_offsets[b + 1]
        kv = length if max_kv is None else min(length, max_kv)
        slots = [page_table[b][s] for s in range(-(-kv // page_size))]
        held = np.array([0 <= slots[p // page_size] < num_pages for p in range(kv)], dtype=bool)
        at = [(slots[p // page_size], p % page_size) for p in range(kv)]
        for h in range(kv_heads):
            key, value = (np.array([VALUES[cache[n][pg, h, r]] * float(cache[n + "_scale"][pg, h]) if ok else np.zeros(dim)
                                    for (pg, r), ok in zip(at, held)]).reshape(kv, dim) for n in "kv")
            for t in range(lo, hi if max_q is None else min(hi, lo + max_q)):
                pos, p = length - (hi - lo) + t - lo, np.arange(kv)
                sees = held.copy()
                if causal:
                    sees &= p <= pos
                if window:
                    sees &= pos - p < window
                if not sees.any():
                    continue
                for g in range(h * (heads // kv_heads), (h + 1) * (heads // kv_heads)):
                    s = scale * (key[sees] @ q[t, g])
                    w = np.exp(s - s.max())
                    lse[t, g] = s.max() + math.log(w.sum())
                    out[t, g], absolute[t, g] = w @ value[sees] / w.sum(), w @ np.abs(value[sees]) / w.sum()
                    spread[t, g] = abs(scale) * (np.abs(key[sees]) @ np.abs(q[t, g])).max()
    return out, lse, absolute, spread


def sample(row, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Sums run in numpy's longdouble, so that none of them is off by as much as a 64-bit rounding."""
    row = np.where(np.isnan(row), -np.inf, np.asarray(row, dtype=np.float64))
    order = sorted(np.flatnonzero(row > -np.inf).tolist(), key=lambda i: (-row[i], i))
    if not order:
        return -1, -math.inf
    if temperature <= 0:
        return order[0], 0.0
    if top_k > 0:
        order = order[:top_k]
    top = row[order[0]]
    w = [1.0 if row[i] == top else 0.0 if top == math.inf else math.exp((row[i] - top) / temperature) for i in order]
    if top_p < 1:
        mass = np.cumsum(np.array(w, dtype=np.longdouble))
        n = 1
        while n < len(w) and mass[n - 1] < top_p * mass[-1]:
            n += 1
        order, w = order[:n], w[:n]
    kept = sorted((i, x) for n, (i, x) in enumerate(zip(order, w)) if n == 0 or x >= min_p)
    mass = np.cumsum(np.array([x for _, x in kept], dtype=np.longdouble))
    at = next((n for n in range(len(kept)) if mass[n] > u * mass[-1]), len(kept) - 1)
    return kept[at][0], math.log(kept[at][1] / mass[-1])
