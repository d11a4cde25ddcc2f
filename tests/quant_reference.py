"""Plain fp64 statements of the quantised cache, and the error that a correct
fp32 computation may have -- test infrastructure.

What is held is exact: the bits of a group follow from its values alone. Bounds of
attention count roundings, as tests/weight_reference.py does, u = 2^-24 being half
a step of fp32. The products of held values (at most 4 significant bits) with bf16
queries, and with each of the three bf16 pieces of an fp32 query, are exact; their
d (3 d) sums round: a logit is off by dx = (d + 4) u X, ((3 d + 4) u X), X = sum_c
|q_c k_c| / sqrt(d), and a probability by rel = 2 dx + (n + 64 + 4 max |x|) u of
itself. An output is off by rel A, A = sum_j a_j |v_j|. In a bf16 cache the two
bf16 pieces of a probability leave 2^-15 of it (less than 2^-7 after the first, of
which the second is off by half a step, 2^-8), and the output is rounded, 2^-8 of
its size. In calls of more than 16 rows per KV head a probability of a bf16 cache is
one fp16 instead, off by half a step, 2^-11 of it, or, below 2^-14 of a unit that
is at most 2^-7 of the largest (2^-21 of it), by 2^-25 of that unit: 2^-32 of the
largest; the values beside it are exact. In an fp32 cache three pieces leave nothing, and their 3 n sums round."""
from __future__ import annotations

import math

import numpy as np

from weight_reference import U32, softmax_error


def values(bits):
    """The magnitudes of the type, in order: those in even places have even codes."""
    if bits == 4:
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    v = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)]
    return np.array(v[:-1])  # the last code is NaN


def held(x, bits):
    """What the cache holds for x [..., d]."""
    grid = values(bits)
    limit, least, most = (7.0, -111, 125) if bits == 4 else (464.0, -111, 119)
    g = np.asarray(x, np.float64)
    g = g.reshape(g.shape[:-1] + (-1, 32))
    top = np.abs(g).max(-1, keepdims=True)
    with np.errstate(all="ignore"):
        e = np.where(np.isfinite(top) & (top > 0), np.floor(np.log2(np.where(top > 0, top, 1.0) / limit)) + 1, least)
        # (the logarithm may be off next to a power of two)
        e = np.where(np.isfinite(e), e, least)
        e = np.where(top >= limit * 2.0 ** e, e + 1, e)
        e = np.where((top < limit * 2.0 ** (e - 1)), e - 1, e)
        X = 2.0 ** np.clip(e, least, most)
        y = np.abs(g) / X
        y = np.where(np.isfinite(y), y, 0.0)
    hi = np.minimum(np.searchsorted(grid, y), len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    below, above = y - grid[lo], grid[hi] - y
    place = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    r = np.copysign(grid[place], g) * X
    r = np.where(np.isfinite(top), r, np.nan)
    return r.reshape(r.shape[:-2] + (-1,))


def attention(q, K, V, bf16, prefix=None, half=False):
    """(out, bound, lse, bound) of q [rows][d] over held K, V [n][d] (n may be 0) and a
    prefix's; half: probabilities are fp16."""
    if prefix is not None:
        K, V = np.concatenate([K, prefix[0]]), np.concatenate([V, prefix[1]])
    rows, d = q.shape
    if len(K) == 0:
        return np.zeros((rows, d)), np.zeros((rows, d)), np.full(rows, -np.inf), np.zeros(rows)
    x = q @ K.T / math.sqrt(d)
    X = (np.abs(q) @ np.abs(K).T).max(axis=1) / math.sqrt(d)
    dx = ((d if bf16 else 3 * d) + 4) * U32 * X
    m = x.max(axis=1, keepdims=True)
    e = np.exp(x - m)
    z = e.sum(axis=1, keepdims=True)
    a = e / z
    rel = softmax_error(dx, x) + (0.0 if bf16 else 2 * len(K) * U32)
    out, A = a @ V, a @ np.abs(V)
    bound = rel[:, None] * A + 2 * U32 * np.abs(out) + 1e-37
    if bf16:
        bound = bound + (2.0 ** -11 * A + 2.0 ** -32 * a.max(axis=1, keepdims=True) * np.abs(V).sum(axis=0) if half
                         else 2.0 ** -15 * A)
        bound = bound + 2.0 ** -8 * (np.abs(out) + bound)
    lse = (m + np.log(z))[:, 0]
    return out, bound, lse, rel + 8 * U32 * (np.abs(lse) + np.log(z)[:, 0] + 1.0)
