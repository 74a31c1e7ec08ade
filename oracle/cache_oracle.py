"""Oracle of the paged cache of keys and values in mx4 and of the attention over it: numpy, 64 bits, whole numbers by plain loops.

A record of 32 positions of a head of D (64, 128 or 256) elements: key codes [32][D/2], value codes [4][16][8][D/32], key scales [32][D/32],
value scales [4][D/32][8]; of the values part (g, m, i) is position 4g + i (i < 4) or 12 + 4g + i, elements m D/16 and following.
"""
from __future__ import annotations

import numpy as np

from . import mx4_oracle as mo

LEAST, MOST = -23, 13                                           # exponents of a scale


def filled(dim):
    return 64 if dim <= 64 else 128 if dim <= 128 else 256


def _ceil(a, b):
    return -(-a // b)


def codes(k, v):
    """Codes (0..15) and scale bytes of the key and the value of one position and head, filled up."""
    out = []
    bad = not (np.isfinite(k).all() and np.isfinite(v).all())
    for is_key, x in ((True, k), (False, v)):
        full = filled(len(x))
        b = np.zeros(full)
        if not bad:
            b[:len(x)] = x
        b = b.reshape(-1, 32)
        amax = np.abs(b).max(-1)
        e = np.where(amax > 0, np.frexp(np.where(amax > 0, amax, 1.0))[1] - 3, 0).clip(LEAST, MOST)
        m = np.abs(b) / np.exp2(e)[:, None]
        dist = np.abs(np.minimum(m, 8.0)[..., None] - np.array(mo.GRID))
        near = dist == dist.min(-1, keepdims=True)
        code = np.where(near[..., 0::2].any(-1), 2 * near[..., 0::2].argmax(-1), 2 * near[..., 1::2].argmax(-1) + 1)
        code = code + 8 * np.signbit(b)
        byte = e + 127
        if bad:
            code, byte = np.zeros_like(code), np.full_like(byte, 255 if is_key else 127)
        out += [code.reshape(-1), byte]
    return out


def place(t):
    """(g, i) of position t of a record among the values."""
    return t % 16 // 4, t % 4 + 4 * (t // 16)


def store(cache, k, v, slots):
    """k, v [tokens, heads, dim] into cache u8 [pages, heads, page/32, 34 D] at slots (those outside are left out)."""
    pages, heads, records, size = cache.shape
    page, full = records * 32, size // 34
    unit = full // 16
    for row, slot in enumerate(slots):
        if not 0 <= slot < pages * page:
            continue
        for h in range(heads):
            kc, ks, vc, vs = codes(k[row, h].astype(np.float64), v[row, h].astype(np.float64))
            t = slot % 32
            r = cache[slot // page, h, slot % page // 32]
            g, i = place(t)
            r[t * full // 2:(t + 1) * full // 2] = kc[0::2] | kc[1::2] << 4
            packed = (vc[0::2] | vc[1::2] << 4).reshape(16, unit // 2)
            r[16 * full:32 * full].reshape(4, 16, 8, unit // 2)[g, :, i] = packed
            r[32 * full:33 * full].reshape(32, full // 32)[t] = ks
            r[33 * full:].reshape(4, full // 32, 8)[g, :, i] = vs


def load(cache, slots, dim):
    """fp64 keys and values [tokens, heads, dim] behind slots; zeros for those outside."""
    pages, heads, records, size = cache.shape
    page, full = records * 32, size // 34
    k, v = np.zeros((len(slots), heads, dim)), np.zeros((len(slots), heads, dim))
    grid = mo.VALUES

    def value(b, s):
        x = np.empty(full)
        x[0::2], x[1::2] = grid[b & 15], grid[b >> 4]
        s = s.astype(np.int64)
        return (x.reshape(-1, 32) * np.where(s == 255, np.nan, np.exp2(np.where(s == 255, 0, s - 127.0)))[:, None]).reshape(-1)[:dim]
    for row, slot in enumerate(slots):
        if not 0 <= slot < pages * page:
            continue
        t = slot % 32
        g, i = place(t)
        for h in range(heads):
            r = cache[slot // page, h, slot % page // 32]
            k[row, h] = value(r[t * full // 2:(t + 1) * full // 2], r[32 * full:33 * full].reshape(32, -1)[t])
            v[row, h] = value(r[16 * full:32 * full].reshape(4, 16, 8, -1)[g, :, i].reshape(-1), r[33 * full:].reshape(4, -1, 8)[g, :, i])
    return k, v


def reserve(held, added, page, table, free, count, tokens):
    """Results of adadim_cache_reserve as a dict; table is a copy."""
    n, table = len(held), table.copy()
    width = table.shape[1]
    slots, positions = [], []
    stack = list(free[:count])
    refused = any(h < 0 or a < 0 or h + a > width * page for h, a in zip(held, added)) or sum(added) > tokens
    need = 0 if refused else sum(_ceil(h + a, page) - _ceil(h, page) for h, a in zip(held, added))
    ok = not refused and need <= count
    offsets = [0]
    for s in range(n):
        if ok:
            for p in range(_ceil(held[s], page), _ceil(held[s] + added[s], page)):
                table[s, p] = stack.pop()
            for pos in range(held[s], held[s] + added[s]):
                positions.append(pos)
                slots.append(int(table[s, pos // page]) * page + pos % page)
        offsets.append(len(slots))
    fill = [-1] * (tokens - len(slots))
    return {"table": table, "lengths": [h + a if ok else h for h, a in zip(held, added)], "offsets": offsets, "slots": slots + fill,
            "positions": positions + fill, "left": len(stack), "lacking": -1 if refused else 0 if ok else need - count}


def trim(held, kept, page, table, free, count):
    free, width = list(free), table.shape[1]
    lengths = []
    for s in range(len(held)):
        h = min(max(held[s], 0), width * page)
        k = min(max(kept[s], 0), h)
        for p in range(_ceil(k, page), _ceil(h, page)):
            if count < len(free):
                free[count] = int(table[s, p])
                count += 1
        lengths.append(k)
    return {"free": free, "lengths": lengths, "left": count}


def attention(q, cache, table, offsets, lengths, dim, scale, causal=True, window=0):
    """q [tokens, query heads, dim].  Returns fp64 (y, weight, slack) of q's shape: the result, sum_j w_j |v_j| of its terms, and what one part in
    one of the scores' own error is worth, max_j scale |q| . |k_j| (NaN rows in no sequence)."""
    pages, heads, records, _ = cache.shape
    page, group = records * 32, q.shape[1] // heads
    y, weight, slack = (np.full(q.shape, np.nan) for _ in range(3))
    for s in range(len(lengths)):
        o0, o1 = (min(max(int(o), 0), len(q)) for o in offsets[s:s + 2])
        length = min(max(int(lengths[s]), 0), table.shape[1] * page)
        ids = table[s][np.arange(length) // page]
        there = (ids >= 0) & (ids < pages)
        k, v = load(cache, np.where(there, ids.astype(np.int64) * page + np.arange(length) % page, -1), dim)
        for row in range(o0, o1):
            pos = length - (o1 - o0) + row - o0
            j = np.arange(length)
            seen = there & (j <= pos if causal else True) & (j > pos - window if window else True)
            for h in range(q.shape[1]):
                if not seen.any():
                    y[row, h], weight[row, h], slack[row, h] = 0, 0, 0
                    continue
                kk, vv = k[seen, h // group], v[seen, h // group]
                score = scale * (kk @ q[row, h])
                p = np.exp(score - np.max(score)) if np.isfinite(score).all() else np.full(len(score), np.nan)
                p = p / p.sum()
                y[row, h], weight[row, h] = p @ vv, p @ np.abs(vv)
                slack[row, h] = scale * (np.abs(kk) @ np.abs(q[row, h])).max()
    return y, weight, slack
