"""Oracle of the selection of experts and of e4m3 operands with a scale per block of 128 -- TEST INFRASTRUCTURE ONLY.

Plain numpy in 64 bits, written from the definitions in include/moe.h; it shares nothing with the library's kernels.

    select      experts and weights of every row of logits
    quantize    e4m3 numbers (as 64-bit values, NaN where an element is not finite) and scale bytes
    value       what quantised rows or matrices stand for
    gemm        the grouped product, and for each result the sum of the products' absolute values, which error bounds are relative to
    ffn         the experts' feed-forward, and a bound for what errors of the first product can move through the second quantisation
"""
from __future__ import annotations

import numpy as np


def select(logits, k, bias=None, score="sigmoid", n_groups=1, groups_kept=1, group_top=2, renormalize=True, scale=1.0):
    """-> idx [T, k], w [T, k] in 64 bits."""
    logits = np.asarray(logits, dtype=np.float64)
    T, E = logits.shape
    size = E // n_groups
    idx, out = np.zeros((T, k), dtype=np.int32), np.zeros((T, k))
    for t in range(T):
        l = np.where(np.isnan(logits[t]), -np.inf, logits[t])
        if score == "sigmoid":
            with np.errstate(over="ignore"):
                s = 1.0 / (1.0 + np.exp(-l))
        else:
            top = l.max()
            if top == -np.inf:
                s = np.zeros(E)
            else:
                e = (l == np.inf).astype(np.float64) if top == np.inf else np.exp(l - top)
                s = e / e.sum()
        key = s + (np.zeros(E) if bias is None else np.asarray(bias, dtype=np.float64))
        key = np.where((l == -np.inf) | np.isnan(key), -np.inf, key)
        s = np.where(key == -np.inf, 0.0, s)
        allowed = np.ones(E, dtype=bool)
        if groups_kept < n_groups:
            of_group = []
            for g in range(n_groups):
                best = sorted((v for v in key[g * size:(g + 1) * size] if v > -np.inf), reverse=True)[:group_top]
                of_group.append(sum(best) if best else -np.inf)
            kept = sorted(range(n_groups), key=lambda g: (-of_group[g], g))[:groups_kept]
            allowed = np.isin(np.arange(E) // size, kept)
        order = sorted(np.flatnonzero(allowed).tolist(), key=lambda e: (-key[e], e))[:k]
        w = s[order]
        if renormalize and w.sum() > 0:
            w = w / w.sum()
        idx[t], out[t] = order, w * scale
    return idx, out


def e4m3(x):
    """The nearest e4m3 numbers of |x| <= 448 (ties to even); NaN stays."""
    x = np.asarray(x, dtype=np.float64)
    _, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
    step = np.ldexp(1.0, np.maximum(e, -5) - 4)
    return np.round(x / step) * step


def scale_exponent(largest):
    """The smallest n >= -126 with largest <= 448 * 2^n; 0 for 0."""
    n = -126
    while largest > 448.0 * 2.0 ** n:
        n += 1
    return n if largest > 0 else 0


def quantize(x, block_rows=1):
    """x [rows, cols] -> numbers [rows, cols], bytes [rows or blocks, columns in groups of four]."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    number = np.empty_like(x)
    scale = np.full((-(-rows // block_rows), -(-cols // 512) * 4), 127, dtype=np.uint8)
    for r in range(0, rows, block_rows):
        for b in range(-(-cols // 128)):
            tile = x[r:r + block_rows, 128 * b:128 * b + 128]
            finite = np.isfinite(tile)
            n = scale_exponent(np.abs(tile[finite]).max() if finite.any() else 0.0)
            scale[r // block_rows, b] = n + 127
            number[r:r + block_rows, 128 * b:128 * b + 128] = e4m3(np.where(finite, tile / 2.0 ** n, np.nan))
    return number, scale


def value(number, scale, block_rows=1):
    rows, cols = number.shape
    s = np.ldexp(1.0, scale.astype(np.int64) - 127)
    return np.asarray(number, dtype=np.float64) * np.repeat(np.repeat(s, block_rows, 0)[:rows], 128, 1)[:, :cols]


def gemm(a, w, offsets, a_rows=None):
    """a [rows, K], w [E, N, K] in 64 bits -> (results, sums of absolute values) of the rows that an expert has; 0 elsewhere."""
    rows = len(a) if a_rows is None else len(a_rows)
    out, size = np.zeros((rows, w.shape[1])), np.zeros((rows, w.shape[1]))
    for e in range(len(offsets) - 1):
        r = np.arange(offsets[e], offsets[e + 1])
        x = a[r if a_rows is None else np.asarray(a_rows)[r]]
        out[r], size[r] = x @ w[e].T, np.abs(x) @ np.abs(w[e]).T
    return out, size


def moved(h, delta):
    """How far quantised rows of h may move where every element may be off by delta: the larger way, element by element."""
    low, high = np.empty_like(h), np.empty_like(h)
    far = np.zeros_like(h)
    for b in range(0, h.shape[1], 128):
        tile, d = h[:, b:b + 128], delta[:, b:b + 128]
        for r in range(len(h)):
            most = np.abs(tile[r])
            centre = 2.0 ** scale_exponent(most.max())
            at = e4m3(tile[r] / centre) * centre
            # the scale may be that of the smallest and that of the largest maximum
            for largest in {scale_exponent((most - d[r]).max()) if (most - d[r]).max() > 0 else -126, scale_exponent((most + d[r]).max())}:
                s = 2.0 ** largest
                for sign in (-1.0, 1.0):
                    to = e4m3(np.clip((tile[r] + sign * d[r]) / s, -448, 448)) * s
                    far[r, b:b + 128] = np.maximum(far[r, b:b + 128], np.abs(to - at))
    return far


def ffn(x, w1, w2, offsets, activation, src_tok=None, sum_error=0.0):
    """x [rows, D] as its quantised rows' values, w1 [E, 2, F, D] (silu) or [E, F, D], w2 [E, D, F] in 64 bits; sum_error: what a sum may be
    off by, relative to the sum of its products' absolute values -> (y, bound): the exact results of these definitions, and how far
    sums that are off by so much may move them."""
    if activation == "silu":
        g, g_size = gemm(x, w1[:, 0], offsets, src_tok)
        u, u_size = gemm(x, w1[:, 1], offsets, src_tok)
        with np.errstate(over="ignore"):
            s = g / (1.0 + np.exp(-g))
        h = s * u
        # |silu'| <= 1.1; the exponential and the division in fp32 are off by some 2^-24 of |g| + 4
        ds = 1.1 * sum_error * g_size + np.abs(s) * (np.abs(g) + 4.0) * 2.0 ** -23
        du = sum_error * u_size
        delta = ds * np.abs(u) + np.abs(s) * du + ds * du + 2.0 ** -23 * np.abs(h)
    else:
        g, g_size = gemm(x, w1, offsets, src_tok)
        h, delta = np.maximum(g, 0.0), sum_error * g_size
    number, scale = quantize(h)
    q = value(number, scale)
    y, y_size = gemm(q, w2, offsets)
    far, _ = gemm(moved(h, delta), np.abs(w2), offsets)
    return y, far + sum_error * (y_size + far)
