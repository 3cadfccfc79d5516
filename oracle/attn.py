"""fp64 reference of decoding on a translated cache (test infrastructure).

Plain numpy, one row and head at a time, from the definitions: rotary
positions by complex multiplication, masked softmax attention over the slots
of a context, column sums of its weights, and selection by sorting.  Caches
are given as contiguous rows per context; the tests do the paging.
"""
from __future__ import annotations

import numpy as np


def rotate(x, pos, freq, axis):
    """Rotate-half RoPE of x [rows, heads, D]: pair (e, e + D/2) of a row turns
    by pos[axis[e]][row] * freq[e]."""
    half = x.shape[-1] // 2
    ang = np.asarray(pos, np.float64)[np.asarray(axis)].T * np.asarray(freq, np.float64)
    z = (x[..., :half] + 1j * x[..., half:]) * np.exp(1j * ang)[:, None, :]
    return np.concatenate([z.real, z.imag], axis=-1)


def visible(p, n, window, prefix):
    """Slots that the new token of slot p sees, as a mask over [0, n)."""
    j = np.arange(n)
    if p < 0:
        return np.zeros(n, bool)
    see = (j <= p) | (j < prefix)
    if window:
        see &= j > p - window
    return see


def _scores(q, k, scale, cap):
    s = scale * (k @ q)
    return cap * np.tanh(s / cap) if cap else s


def attend(q, k, v, scale, cap=0.0, window=0, prefix=0):
    """One context: q [m, Hq, D], k and v [n, Hkv, D].  Returns out
    [m, Hq, D], lse [m, Hq], the weights' sum of magnitudes sum_j p_j |v_j|
    [m, Hq, D] (what a relative error of the weights is measured on) and the
    largest sum of |q k| * scale behind a visible score [m, Hq]."""
    m, hq, d = q.shape
    n, hkv, _ = k.shape
    out, mag = np.zeros((m, hq, d)), np.zeros((m, hq, d))
    lse, size = np.full((m, hq), -np.inf), np.zeros((m, hq))
    for i in range(m):
        see = visible(n - m + i, n, window, prefix)
        if not see.any():
            continue
        for h in range(hq):
            kh, vh = k[see, h // (hq // hkv)], v[see, h // (hq // hkv)]
            s = _scores(q[i, h], kh, scale, cap)
            top = s.max()
            e = np.exp(s - top)
            w = e / e.sum()
            out[i, h] = w @ vh
            mag[i, h] = w @ np.abs(vh)
            lse[i, h] = top + np.log(e.sum())
            size[i, h] = scale * (np.abs(kh) @ np.abs(q[i, h])).max()
    return out, lse, mag, size


def mass(q, k, lse, scale, cap=0.0, window=0, prefix=0):
    """One context: weight [Hkv, n] that the slots receive, and the largest
    sum of |q k| * scale behind a visible score."""
    m, hq, _ = q.shape
    n, hkv, _ = k.shape
    got, size = np.zeros((hkv, n)), 0.0
    for i in range(m):
        see = visible(n - m + i, n, window, prefix)
        if not see.any():
            continue
        for h in range(hq):
            kh = k[see, h // (hq // hkv)]
            got[h // (hq // hkv), see] += np.exp(_scores(q[i, h], kh, scale, cap) - lse[i, h])
            size = max(size, scale * float((np.abs(kh) @ np.abs(q[i, h])).max()))
    return got, size


def keep(weight, keep, sink, recent):
    """Slots kept of one (layer, context, head): weight [n] fp32."""
    n = len(weight)
    if n <= keep:
        return np.arange(n)
    w = np.where(np.isnan(weight), -np.inf, weight.astype(np.float64))
    always = [j for j in range(n) if j < sink or j >= n - recent]
    rest = sorted((j for j in range(n) if sink <= j < n - recent), key=lambda j: (-w[j], j))
    return np.array(sorted(always + rest[:keep - len(always)]), int)
