"""Plain fp64 statements of the weight cache, the shared prefix and the prompt
weights, one unit (sequence and KV head) at a time, with the error that a
correct fp32 computation may have -- test infrastructure.

The bounds count roundings. With u = 2^-24 (half a step of fp32), a logit is a
sum of d exact (bf16) or rounded (fp32) products scaled once: it is off by at
most dx = (d + 4) u X, X = sum_c |q_c k_c| / sqrt(d), at most over the tokens. A
softmax probability a is then off by at most (2 dx + r) a, where r = (n + 64) u
covers the sum of n terms, the exponentials (a few u each, and u times the
logits' size) and the joins. An output is off by (2 dx + r) A, A = sum_j a_j
|v_j|; where values are bf16, the probabilities that multiply them are rounded
to bf16 (half a step: 2^-8 each), and the output is rounded once more."""
from __future__ import annotations

import math

import numpy as np

U32 = 2.0 ** -24
HALF_BF16 = 2.0 ** -8


def logits(q, K):
    """[G][n] scaled logits of q [G][d] over K [n][d], and dx [G]."""
    d = q.shape[1]
    x = q @ K.T / math.sqrt(d)
    X = (np.abs(q) @ np.abs(K).T).max(axis=1, initial=0.0) / math.sqrt(d)
    return x, (d + 4) * U32 * X


def softmax_error(dx, x):
    """Relative error of each head's probabilities."""
    big = np.abs(x).max(axis=1, initial=0.0)
    return 2.0 * dx + (x.shape[1] + 64 + 4.0 * big) * U32


def output_bound(a, V, rel, bf16, ref):
    """Elementwise error of a V [G][d], a [G][n] with relative errors rel [G]."""
    A = a @ np.abs(V)
    b = rel[:, None] * A
    if bf16:
        b = b + HALF_BF16 * A + HALF_BF16 * (np.abs(ref) + 2 * HALF_BF16 * A)
    return b + 2 * U32 * np.abs(ref) + 1e-37


class Unit:
    """One unit of a weight cache: its places in order."""

    def __init__(self, G, d, capacity, recent, bf16):
        self.G, self.d, self.C, self.recent, self.bf16 = G, d, capacity, recent, bf16
        self.start(np.zeros((0, d)), np.zeros((0, d)), None)

    def start(self, K, V, w):
        n, C = len(K), self.C
        w = np.zeros(n) if w is None else np.asarray(w, np.float64)
        pos = np.arange(n)
        if n > C:
            old = sorted(range(n - self.recent), key=lambda p: (w[p], p))
            kept = sorted(old[n - C:]) + list(range(n - self.recent, n))
            pos = np.array(kept)
        self.pos = np.full(C, -1, np.int64)
        self.w, self.err = np.zeros(C), np.zeros(C)
        m = self.n = len(pos)
        self.K, self.V = (np.zeros((min(C, 2 * m + 64), self.d)) for _ in range(2))  # grows in step()
        self.pos[:m], self.w[:m], self.K[:m], self.V[:m] = pos, w[pos], K[pos], V[pos]
        self.clock = n

    def lightest(self, seen):
        """The place of the token to go. Where the one at position `seen` is as
        light within the weights' errors, two correct sums may differ about
        which is the lighter, and it goes."""
        old = [j for j in range(self.C) if self.pos[j] < self.clock - self.recent]
        least = min(old, key=lambda j: (self.w[j], self.pos[j]))
        other = [j for j in old if self.pos[j] == seen]
        if other and other[0] != least and self.w[other[0]] - self.w[least] < self.err[other[0]] + self.err[least]:
            return other[0]
        return least

    def step(self, q, k, v, prefix=None, seen=None):
        """(out, its bound, evicted position or -1); seen: the position that the library evicted."""
        evicted = -1
        place = self.n
        if self.n == self.C:
            place = self.lightest(seen)
            evicted = int(self.pos[place])
        self.n = max(self.n, place + 1)
        if place >= len(self.K):
            self.K, self.V = (np.concatenate([x, np.zeros((min(self.C, 2 * place) + 1 - len(x), self.d))])
                              for x in (self.K, self.V))
        self.pos[place], self.w[place], self.err[place], self.K[place], self.V[place] = self.clock, 0.0, 0.0, k, v
        K, V, n = self.K[:self.n], self.V[:self.n], self.n
        if prefix is not None:
            K, V = np.concatenate([K, prefix[0]]), np.concatenate([V, prefix[1]])
        x, dx = logits(q, K)
        a = np.exp(x - x.max(axis=1, keepdims=True))
        a /= a.sum(axis=1, keepdims=True)
        rel = softmax_error(dx, x)
        out = a @ V
        self.w[:n] += a[:, :n].sum(axis=0)
        self.err[:n] += (rel[:, None] * a[:, :n]).sum(axis=0) + (self.G + 2) * U32 * self.w[:n]
        self.clock += 1
        return out, output_bound(a, V, rel, self.bf16, out), evicted


def prefix_attention(q, K, V, bf16):
    """(out, bound, lse, bound) of q [G][d] over K, V [n][d], n >= 1."""
    x, dx = logits(q, K)
    m = x.max(axis=1, keepdims=True)
    e = np.exp(x - m)
    z = e.sum(axis=1, keepdims=True)
    rel = softmax_error(dx, x)
    out = e / z @ V
    lse = (m + np.log(z))[:, 0]
    return out, output_bound(e / z, V, rel, bf16, out), lse, rel + 8 * U32 * (np.abs(lse) + np.log(z)[:, 0] + 1.0)


def prompt_weights(q, K, prefix_lse=None):
    """(weights, bound) [n]: q [rows][G][d] of the last `rows` tokens, K [n][d], prefix_lse [rows][G]."""
    rows, n = len(q), len(K)
    w, err = np.zeros(n), np.zeros(n)
    for i in range(rows):
        last = n - rows + i + 1
        x, dx = logits(q[i], K[:last])
        m = x.max(axis=1)
        if prefix_lse is not None:
            m = np.maximum(m, prefix_lse[i])
        e = np.exp(x - m[:, None])
        z = e.sum(axis=1) + (0.0 if prefix_lse is None else np.exp(prefix_lse[i] - m))
        a = e / z[:, None]
        off = softmax_error(dx, x)
        if prefix_lse is not None:
            off = off + 8 * U32 * (np.abs(prefix_lse[i]) + 1.0)
        # (the exponent x - lse is rounded once more, at its own size)
        off = off + 4 * U32 * (np.abs(x).max(axis=1) + np.abs(m) + math.log(n + 1.0))
        w[:last] += a.sum(axis=0)
        err[:last] += (off[:, None] * a).sum(axis=0)
    return w, err + (rows * q.shape[1] + 8) * U32 * w + 1e-37
