"""Oracle of routing, plans, grouped products, combining, and norms of queries and keys.

TEST INFRASTRUCTURE ONLY: imported by the test suite, never by the product
library; it shares no code with the GPU path.  Definitions as include/mxq.h
states them, in float64.
"""
from __future__ import annotations

import numpy as np

import oracle
from oracle.paged import to_f32

BLOCK, ROWS = 32, 16


def route(logits, k, score="softmax", normalise=True, scale=1.0, bias=None):
    """(ids int32 [T, k], weights float64 [T, k])."""
    T, E = logits.shape
    ids, w = np.full((T, k), -1, np.int32), np.zeros((T, k))
    for t in range(T):
        x = logits[t].astype(np.float64)
        ok = ~np.isnan(x) & (x != -np.inf)
        x = np.minimum(x, float(np.finfo(np.float32).max))
        if not ok.any():
            continue
        with np.errstate(over="ignore"):
            if score == "softmax":
                s = np.where(ok, np.exp(np.where(ok, x, 0) - x[ok].max()), 0.0)
                s = s / s.sum()
            else:
                s = np.where(ok, 1 / (1 + np.exp(-np.where(ok, x, 0))), 0.0)
        key = x if bias is None else s + bias.astype(np.float64)
        may = ok & ~np.isnan(key) & (key != -np.inf)
        order = [e for e in sorted(range(E), key=lambda e: (-key[e] if may[e] else np.inf, e)) if may[e]][:k]
        got = s[order]
        if normalise and order:                          # ratios, whatever the scores' size
            c = x[order]
            if score == "softmax":
                got = np.exp(c - c.max())
            else:
                low = np.minimum(c, 0)
                got = np.exp(low - min(c.max(), 0)) / (1 + np.exp(-np.abs(c)))
            got = got / got.sum()
        ids[t, :len(order)], w[t, :len(order)] = order, got * np.float64(np.float32(scale))
    return ids, w


def rows_of(pairs, experts):
    return (pairs + (ROWS - 1) * min(pairs, experts)) // ROWS * ROWS


def plan(ids, experts):
    """(first int32 [E + 1], pair int32 [rows])."""
    f = np.asarray(ids).reshape(-1)
    first, pair = np.zeros(experts + 1, np.int32), np.full(rows_of(f.size, experts), -1, np.int32)
    for e in range(experts):
        here = np.nonzero(f == e)[0]
        pair[first[e]:first[e] + len(here)] = here
        first[e + 1] = first[e] + (len(here) + ROWS - 1) // ROWS * ROWS
    return first, pair


def product(bits, w_bits, ids, perms, widths, round_mode=0, clamp_mode=0):
    """bits [pairs, K], w_bits [E, N, K], perms [K], [E, K] or None: (y, bound) float64
    [pairs, N], NaN where no expert is chosen; bound: what the sums' terms add up to in
    absolute value, with the digits that an m-bit mantissa is split into."""
    f = np.asarray(ids).reshape(-1)
    E, N, _ = w_bits.shape
    y, big = np.full((f.size, N), np.nan), np.zeros((f.size, N))
    # |8 h| + |l| <= |q| + 14 (6 bits), |16 h| + |l| <= |q| + 30 (8 bits)
    more = np.repeat([{3: 0, 4: 0, 6: 14, 8: 30}[m] for m in widths], BLOCK)
    for e in range(E):
        here = np.nonzero(f == e)[0]
        if not len(here):
            continue
        p = None if perms is None else perms if perms.ndim == 1 else perms[e]
        sides = []
        for x in (bits[here], w_bits[e]):
            q, ex = oracle.quantize(x, perm=p, widths=widths, round_mode=round_mode, clamp_mode=clamp_mode)
            unit = np.exp2(ex.astype(np.float64) - 127 - (np.asarray(widths) - 2)).repeat(BLOCK, axis=1)
            sides.append((oracle.dequantize(q, ex, widths), (np.abs(q.astype(np.float64)) + more) * unit,
                          (ex == 255).any(axis=1)))
        (a, aa, an), (w, ww, wn) = sides
        y[here], big[here] = a @ w.T, aa @ ww.T
        y[np.ix_(here[an], range(N))] = np.nan
        y[np.ix_(here, np.nonzero(wn)[0])] = np.nan
    return y, big


def combine(y, ids, weights, experts, residual=None):
    """y float64 [pairs, N] -> (out, bound) float64 [T, N]."""
    T, k = ids.shape
    out = np.zeros((T, y.shape[1])) if residual is None else residual.astype(np.float64).copy()
    big = np.abs(out)
    for t in range(T):
        for j in range(k):
            if 0 <= ids[t, j] < experts:
                term = float(weights[t, j]) * y[t * k + j]
                out[t] += term
                big[t] += np.abs(term)
    return out, big


def norm_rope(bits, pos, table, gain_bits, eps, interleaved):
    """bits uint16 [T, H, D] -> (y, bound) float64: bound is what a relative error of
    every normalised value moves a result by."""
    x = to_f32(bits).astype(np.float64)
    P, half, _ = table.shape
    m = (x * x).mean(-1, keepdims=True) + np.float64(np.float32(eps))
    v = np.where(m == 0, 0.0, x / np.sqrt(np.where(m == 0, 1.0, m))) * to_f32(gain_bits).astype(np.float64)
    y, big = v.copy(), np.abs(v)
    for t in range(x.shape[0]):
        i = np.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        if not 0 <= pos[t] < P:
            y[t][:, np.concatenate([a, b])] = np.nan
            continue
        c, s = table[pos[t], :, 0].astype(np.float64), table[pos[t], :, 1].astype(np.float64)
        y[t][:, a], y[t][:, b] = v[t][:, a] * c - v[t][:, b] * s, v[t][:, b] * c + v[t][:, a] * s
        big[t][:, a] = np.abs(v[t][:, a] * c) + np.abs(v[t][:, b] * s)
        big[t][:, b] = np.abs(v[t][:, b] * c) + np.abs(v[t][:, a] * s)
    return y, big
