"""fp64 reference of serving on caches of 8 bits, with sinks and drafted trees
(test infrastructure).

Plain numpy from the definitions: codes by searching the powers of two and the
nearest code, what a row sees as a mask over its context's slots, and softmax
attention over it one row and head at a time.
"""
from __future__ import annotations

import numpy as np


def _e4m3():
    """The numbers that codes 0..126 stand for, rising."""
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e > 0, (8 + m) * 2.0 ** (e - 10), m * 2.0 ** -9)


E4M3 = _e4m3()
MOST = {"i8": 127.0, "e4m3": 448.0}


def encode(x, code):
    """(codes as bytes, scales) of rows x [..., D]: the smallest power of two,
    from 2^-100 on, that brings a row to the largest code, and the nearest codes,
    ties to even ones.  Rows with a number that is not finite: codes 0, scale NaN."""
    x = np.asarray(x, np.float64)
    odd = ~np.isfinite(x).all(-1)
    x = np.where(odd[..., None], 0.0, np.clip(x, -2.0 ** 127, 2.0 ** 127))
    top = np.abs(x).max(-1)
    scale = np.full(top.shape, 2.0 ** -100)
    for e in range(-99, 123):
        scale = np.where(top > MOST[code] * scale, 2.0 ** e, scale)
    y = x / scale[..., None]
    if code == "i8":
        codes = np.rint(y).astype(np.int8).view(np.uint8)
    else:
        a = np.abs(y)
        hi = np.clip(np.searchsorted(E4M3, a), 0, 126)
        lo = np.maximum(hi - 1, 0)
        up, down = E4M3[hi] - a, a - E4M3[lo]
        codes = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
        codes = (codes | np.where(np.signbit(y), 128, 0)).astype(np.uint8)
    return np.where(odd[..., None], 0, codes).astype(np.uint8), np.where(odd, np.nan, scale)


def decode(codes, scale, code):
    """The numbers that codes (bytes) and scales stand for."""
    c = np.asarray(codes, np.uint8)
    if code == "i8":
        x = c.view(np.int8).astype(np.float64)
    else:
        x = np.append(E4M3, np.nan)[c & 127] * np.where(c & 128, -1.0, 1.0)
    return x * np.asarray(scale, np.float64)[..., None]


def sight(m, n, window=0, sink=0, prefix=0):
    """[m, n]: which slots the new tokens see."""
    see = np.zeros((m, n), bool)
    for i in range(m):
        p = n - m + i
        for j in range(n if p >= 0 else 0):
            see[i, j] = (j <= p or j < prefix) and (window == 0 or j > p - window or j < sink)
    return see


def paths(parents):
    """Every node's path, itself first."""
    out = []
    for i in range(len(parents)):
        path, k = [], i
        while k >= 0:
            path.append(k)
            k = parents[k] if parents[k] < k else -1
        out.append(path)
    return out


def tree_sight(parents, n, window=0, sink=0):
    """[m, n] of a tree's nodes, and their depths."""
    m, see = len(parents), np.zeros((len(parents), n), bool)
    up = paths(parents)
    for i, path in enumerate(up):
        if n - m + i < 0:
            continue
        p = n - m + len(path) - 1
        for j in range(max(n - m, 0)):
            see[i, j] = window == 0 or j > p - window or j < sink
        for before, k in enumerate(path):
            if n - m + k >= 0:
                see[i, n - m + k] = window == 0 or before < window or p - before < sink
    return see, [len(p) - 1 for p in up]


def attend(q, k, v, see, scale, cap=0.0):
    """One context: q [m, Hq, D], k and v [n, Hkv, D], see [m, n]; returns what
    attn.attend does."""
    m, hq, d = q.shape
    hkv = k.shape[1]
    out, mag = np.zeros((m, hq, d)), np.zeros((m, hq, d))
    lse, size = np.full((m, hq), -np.inf), np.zeros((m, hq))
    for i in range(m):
        if not see[i].any():
            continue
        for h in range(hq):
            kh, vh = k[see[i], h // (hq // hkv)], v[see[i], h // (hq // hkv)]
            s = scale * (kh @ q[i, h])
            if cap:
                s = cap * np.tanh(s / cap)
            top = s.max()
            e = np.exp(s - top)
            w = e / e.sum()
            out[i, h] = w @ vh
            mag[i, h] = w @ np.abs(vh)
            lse[i, h] = top + np.log(e.sum())
            size[i, h] = scale * (np.abs(kh) @ np.abs(q[i, h])).max()
    return out, lse, mag, size
