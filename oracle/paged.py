"""Oracle of rotary positions, the paged MXINT KV cache and attention over it.

TEST INFRASTRUCTURE ONLY: imported by the test suite, never by the product
library; it shares no code with the GPU path.

Definitions (include/mxq.h).  Rotation: each pair (x1, x2) of a head becomes
(x1 c - x2 s, x2 c + x1 s) in float32, every operation rounded on its own, then
bf16.  Pages: per KV head and 32-value block a plane of page_tokens packed
blocks.  Attention, in float64: scores over the visible tokens, softmax, the
values' mean; a row that sees nothing is zero.
"""
from __future__ import annotations

import numpy as np

import oracle

D, BLOCK = 128, 32


def to_f32(bits):
    return (np.asarray(bits, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32)


def to_bf16(x):
    """float32 -> bf16 bits, round-to-nearest-even; any NaN is 0xFFFF."""
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0xFFFF), r)


def rope(bits, pos, table, interleaved):
    """bits uint16 [T, H, D], pos [T], table float32 [P, rot / 2, 2]."""
    P, half, _ = table.shape
    x = to_f32(bits)
    out = np.array(bits, dtype=np.uint16)
    for t in range(x.shape[0]):
        ok = 0 <= pos[t] < P
        c, s = (table[pos[t], :, 0], table[pos[t], :, 1]) if ok else (None, None)
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            if not ok:
                out[t, :, a] = out[t, :, b] = 0xFFFF
                continue
            u, v = x[t, :, a], x[t, :, b]
            with np.errstate(all="ignore"):
                out[t, :, a] = to_bf16(u * c[i] - v * s[i])
                out[t, :, b] = to_bf16(v * c[i] + u * s[i])
    return out


def place(widths, Hkv, page, slot, head, block):
    """(byte of the block's mantissas, byte of its exponent) in the pool."""
    row = sum(4 * m for m in widths)
    g, i = divmod(slot, page)
    mant = (g * Hkv + head) * page * row + page * sum(4 * m for m in widths[:block])
    return mant + i * 4 * widths[block], ((g * Hkv + head) * page + i) * 4 + block


def append(mant, exp, bits, slots, widths, Hkv, page, pages, round_mode=0, clamp_mode=0):
    """Quantizes bf16 rows [T, Hkv, D] into the pool's bytes (in place)."""
    T = bits.shape[0]
    q, e = oracle.quantize(bits.reshape(T * Hkv, D), widths=widths, round_mode=round_mode,
                           clamp_mode=clamp_mode)
    rows = oracle.pack_act(q, widths)
    for t in range(T):
        if not 0 <= slots[t] < pages * page:
            continue
        for h in range(Hkv):
            at = 0
            for b, m in enumerate(widths):
                pm, pe = place(widths, Hkv, page, int(slots[t]), h, b)
                mant[pm:pm + 4 * m] = rows[t * Hkv + h, at:at + 4 * m]
                exp[pe] = e[t * Hkv + h, b]
                at += 4 * m


def values(bits, widths, round_mode=0, clamp_mode=0):
    """The float64 values that quantized bf16 rows [..., D] stand for."""
    q, e = oracle.quantize(bits.reshape(-1, D), widths=widths, round_mode=round_mode,
                           clamp_mode=clamp_mode)
    w = np.repeat(np.asarray(widths), BLOCK)
    E = np.repeat(e[:, :len(widths)].astype(np.int64), BLOCK, axis=1)
    return np.ldexp(q.astype(np.float64), E - 127 - (w - 2)).reshape(bits.shape)


def visible(p, n, window, prefix):
    j = np.arange(n)
    see = j <= p
    if window:
        see &= p - j < window
    return see | (j < prefix)


def attention(q, k, v, n_new, scale, softcap=0.0, window=0, prefix=0, slopes=None):
    """One sequence: q float64 [n_new, Hq, D]; k, v float64 [len, Hkv, D].
    Returns (o, the weights' mean of |v|, the largest sum of |q_d k_d| * |scale|,
    the largest |bias| of a visible score)."""
    L, Hkv, _ = k.shape
    Hq = q.shape[1]
    o, a = np.zeros(q.shape), np.zeros(q.shape)
    big = bias = 0.0
    for i in range(n_new):
        p = L - n_new + i
        see = visible(p, L, window, prefix)
        if not see.any():
            continue
        dist = np.abs(p - np.arange(L))[see].astype(np.float64)
        for h in range(Hq):
            kk, vv = k[see, h // (Hq // Hkv)], v[see, h // (Hq // Hkv)]
            x = (kk @ q[i, h]) * scale
            big = max(big, float((np.abs(kk) @ np.abs(q[i, h])).max()) * abs(scale))
            if softcap:
                x = softcap * np.tanh(x / softcap)
            if slopes is not None:
                x = x - float(slopes[h]) * dist
                bias = max(bias, abs(float(slopes[h])) * dist.max())
            w = np.exp(x - x.max())
            w /= w.sum()
            o[i, h], a[i, h] = w @ vv, w @ np.abs(vv)
    return o, a, big, bias
