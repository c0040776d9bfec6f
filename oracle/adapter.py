"""Float64 forms of the dropout and of the low-rank adapters beside a shared layer, from their definitions, row by row of a request.

Independent of the GPU library: the generator is written from its publication (Salmon, Moraes, Dror, Shaw: "Parallel random
numbers: as easy as 1, 2, 3", 2011), the products are numpy's.
"""
from __future__ import annotations

import numpy as np


def philox4x32(counter, key, rounds=10):
    """Philox4x32 of uint32 counters [..., 4] under a key of two words; uint32 [..., 4]."""
    c = [np.asarray(counter[..., i], np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    low, s = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(rounds):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> s) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> s) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1).astype(np.uint32)


def threshold(p):
    return int(np.floor(p * 65536 + 0.5))


def keep_mask(rows, channels, p, seed, offset, first=0):
    """True where an element of a row-major [rows][channels] tensor (its first element numbered `first`) is kept."""
    e = np.arange(first, first + rows * channels, dtype=np.uint64)
    n = e >> np.uint64(3)
    counters, where = np.unique(n, return_inverse=True)
    low, s = np.uint64(0xFFFFFFFF), np.uint64(32)
    offset &= (1 << 64) - 1
    c = np.stack([counters & low, counters >> s, np.full_like(counters, offset & 0xFFFFFFFF), np.full_like(counters, offset >> 32)], -1)
    w = philox4x32(c, (seed & 0xFFFFFFFF, seed >> 32))
    i = (e & np.uint64(7)).astype(np.int64)
    half = (w[where, i // 2] >> (16 * (i % 2)).astype(np.uint32)) & np.uint32(0xFFFF)
    return (half >= threshold(p)).reshape(rows, channels)


def factors(rows, channels, p, seed, offset, first=0):
    """What dropout multiplies each element by: 0 or 1 / (1 - p), p the multiple of 1/65536 that is drawn."""
    t = threshold(p)
    if t == 0:
        return np.ones((rows, channels))
    return keep_mask(rows, channels, p, seed, offset, first) * (65536 / (65536 - t) if t < 65536 else 0.0)


def dropout(x, residual, p, seed, offset, first=0):
    f = factors(*x.shape, p, seed, offset, first)
    y = np.where(f != 0, x, 0.0) * f
    return y if residual is None else residual + y


def requests(row_start, adapter, adapters):
    """(first row, row behind the last, variant or -1) of each request."""
    return [(int(u), int(v), int(a) if 0 <= a < adapters else -1) for u, v, a in zip(row_start[:-1], row_start[1:], adapter) if v > u]


def forward(x, w, bias, a, b, scale, row_start, adapter, relu, f=None):
    """y and t; rows of no request are NaN in both."""
    M, R = x.shape[0], a.shape[1]
    y, t = np.full((M, w.shape[0]), np.nan), np.full((M, R), np.nan)
    xd = x if f is None else np.where(f != 0, x, 0.0) * f
    for u, v, s in requests(row_start, adapter, a.shape[0]):
        y[u:v] = x[u:v] @ w.T + (0 if bias is None else bias)
        t[u:v] = 0
        if s >= 0:
            t[u:v] = xd[u:v] @ a[s].T
            y[u:v] += (1 if scale is None else scale[s]) * (t[u:v] @ b[s].T)
    if relu:
        y = np.where(y < 0, 0.0, y)
    return y, t


def backward(dy, x, w, a, b, scale, row_start, adapter, t, f=None):
    """dx (NaN in rows of no request), da, db."""
    dx = np.full(x.shape, np.nan)
    da, db = np.zeros(a.shape), np.zeros(b.shape)
    xd = x if f is None else np.where(f != 0, x, 0.0) * f
    for u, v, s in requests(row_start, adapter, a.shape[0]):
        dx[u:v] = dy[u:v] @ w
        if s >= 0:
            c = 1 if scale is None else scale[s]
            up = c * (dy[u:v] @ b[s])
            back = up @ a[s]
            dx[u:v] += back if f is None else np.where(f[u:v] != 0, back, 0.0) * f[u:v]
            da[s] += up.T @ xd[u:v]
            db[s] += c * (dy[u:v].T @ t[u:v])
    return dx, da, db
