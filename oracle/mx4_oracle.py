"""Oracle of the microscaled 4-bit operators and of the experts' routing: numpy, 64 bits, from the definitions.

A row is cut into blocks of 32; a block stores the byte e + 127 of a power of two and 32 codes (sign, two bits of exponent,
one of mantissa).  Rows are held in pieces of 128 values: codes u8 [rows, 64 * pieces], scales u8 [pieces, rows, 4].
"""
from __future__ import annotations

import numpy as np

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)                 # magnitude of the code's low three bits
VALUES = np.array(GRID + tuple(-v for v in GRID))


def quantize(x):
    """(codes, scales) of x [rows, cols] (any float type; bfloat16 as float32)."""
    x = np.asarray(x).astype(np.float64)
    rows, cols = x.shape
    pieces = -(-cols // 128)
    b = np.zeros((rows, pieces * 128))
    b[:, :cols] = x
    b = b.reshape(rows, pieces * 4, 32)
    mag = np.abs(b)
    bad = ~np.isfinite(b).all(-1)
    mag = np.where(bad[..., None], 0.0, mag)
    amax = mag.max(-1)
    e = np.where(amax > 0, np.frexp(np.where(amax > 0, amax, 1.0))[1] - 3, 0)      # frexp: amax = m 2^e, m in [1/2, 1)
    e = np.maximum(e, -127)
    m = np.ldexp(mag, -e[..., None])
    dist = np.abs(m[..., None] - np.array(GRID))
    near = dist == dist.min(-1, keepdims=True)
    # of two equally near codes the even one: both are neighbours, so exactly one is
    code = np.where(near[..., 0::2].any(-1), 2 * near[..., 0::2].argmax(-1), 2 * near[..., 1::2].argmax(-1) + 1)
    code = code.astype(np.uint8) | (np.signbit(b).astype(np.uint8) << 3)
    code[bad] = 0
    code = code.reshape(rows, pieces * 128)
    byte = np.where(bad, 255, e + 127).astype(np.uint8)
    return code[:, 0::2] | (code[:, 1::2] << 4), np.ascontiguousarray(byte.reshape(rows, pieces, 4).transpose(1, 0, 2))


def values(codes, scales, cols):
    """fp64 values [rows, cols]."""
    rows = codes.shape[0]
    q = np.empty((rows, codes.shape[1] * 2))
    q[:, 0::2], q[:, 1::2] = VALUES[codes & 15], VALUES[codes >> 4]
    byte = scales.transpose(1, 0, 2).reshape(rows, -1).astype(np.int64)
    s = np.where(byte == 255, np.nan, np.ldexp(1.0, np.where(byte == 255, 0, byte - 127)))
    return (q.reshape(rows, -1, 32) * s[..., None]).reshape(rows, -1)[:, :cols]


def product(w, x):
    """(X W^T, |X| |W|^T) in fp64 of values w [out, in] and x [rows, in]."""
    return x @ w.T, np.abs(x) @ np.abs(w).T


def experts_product(w, x, offsets, rows=None):
    """The same by expert: w [experts, out, in]; rows of Y in no group are NaN in both results."""
    n = len(rows) if rows is not None else x.shape[0]
    y, a = np.full((n, w.shape[1]), np.nan), np.full((n, w.shape[1]), np.nan)
    for e in range(w.shape[0]):
        lo, hi = (int(np.clip(v, 0, n)) for v in offsets[e:e + 2])
        for r in range(lo, hi):
            src = r if rows is None else int(rows[r])
            xr = x[src] if 0 <= src < x.shape[0] else np.zeros(x.shape[1])
            y[r], a[r] = w[e] @ xr, np.abs(w[e]) @ np.abs(xr)
    return y, a


def route(logits, k, renormalize):
    """{chosen, weights, offsets, rows, slots} by plain loops."""
    l = np.asarray(logits).astype(np.float64)
    tokens, experts = l.shape
    chosen, weights = np.full((tokens, k), -1, np.int32), np.zeros((tokens, k))
    for t in range(tokens):
        can = [e for e in range(experts) if l[t, e] > -np.inf]          # false for NaN
        won = sorted(can, key=lambda e: (-l[t, e], e))[:k]
        if not won:
            continue
        top = l[t, won[0]]
        p = {e: 1.0 if l[t, e] == top else float(np.exp(l[t, e] - top)) for e in can}
        total = sum(p[e] for e in (won if renormalize else can))
        for j, e in enumerate(won):
            chosen[t, j], weights[t, j] = e, p[e] / total
    rows, slots, offsets = np.full(tokens * k, -1, np.int32), np.full((tokens, k), -1, np.int32), [0]
    n = 0
    for e in range(experts):
        for t in range(tokens):
            for j in range(k):
                if chosen[t, j] == e:
                    rows[n], slots[t, j] = t, n
                    n += 1
        offsets.append(n)
    return {"chosen": chosen, "weights": weights, "offsets": np.array(offsets, np.int32), "rows": rows, "slots": slots}


def combine(z, slots, weights):
    """(sum, sum of magnitudes) in fp64."""
    z = z.astype(np.float64)
    ok = (slots >= 0) & (slots < z.shape[0])
    y, a = np.zeros((slots.shape[0], z.shape[1])), np.zeros((slots.shape[0], z.shape[1]))
    for t, j in zip(*np.nonzero(ok)):
        term = float(weights[t, j]) * z[slots[t, j]]
        y[t] += term
        a[t] += np.abs(term)
    return y, a
