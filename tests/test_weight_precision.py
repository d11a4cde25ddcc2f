"""How exact the weight cache's step, the shared prefix and the prompt weights
are, on the GPU against 64 bits: bf16 probabilities' halves, logits far from 0.

Bounds. With u = 2^-24 the softmax and the sums are off by rel A, as
tests/weight_reference.py derives it (A = sum_j a_j |v_j|). Beside bf16 values a
probability is the sum of its upper 16 bits, which leave less than 2^-7 of it,
and of that rest rounded to bf16 (half a step, 2^-8): off by 2^-15 of itself, and
an output by 2^-15 A. What is then rounded to bf16 moves by 2^-8 of its size."""
from __future__ import annotations

import numpy as np
import pytest

import weight_reference as ref
from harness import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_11147_amd as raas

    raas.load_library()


def _data(rng, shape):
    import torch

    x = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).bfloat16()
    return x.cuda(), x.double().numpy()


def _np(t):
    return t.detach().double().cpu().numpy()


def _attention(q, K, V):
    """(out, its bound) of q [rows][d] over K, V [n][d], bf16."""
    x, dx = ref.logits(q, K)
    a = np.exp(x - x.max(axis=1, keepdims=True))
    a /= a.sum(axis=1, keepdims=True)
    out, A = a @ V, a @ np.abs(V)
    bound = ref.softmax_error(dx, x)[:, None] * A + 2.0 ** -15 * A + 2 * ref.U32 * np.abs(out)
    return out, bound + 2.0 ** -8 * (np.abs(out) + bound) + 1e-37


def _within(got, want, bound, what):
    over = np.abs(got - want) - bound
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, (what, at, got[at], want[at], bound[at])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [3, 20, 65, 129])  # of G = 2: every prefix kernel
def test_prefix_probabilities(rows, d):
    import torch

    import paper_2502_11147_amd as raas

    say("case precision prefix %d %d" % (rows, d))
    Hq, Hkv, n = 4, 2, 700
    rng = np.random.default_rng(rows)
    (k, K), (v, V), (q, Q) = _data(rng, (Hkv, n, d)), _data(rng, (Hkv, n, d)), _data(rng, (rows, Hq, d))
    p = raas.SharedPrefix(1, Hq, Hkv, d, n, rows, "bf16")
    p.store(0, k, v)
    out = torch.empty_like(q)
    p.attend(0, q, out)
    for h in range(Hkv):
        want, bound = _attention(Q[:, 2 * h:2 * h + 2].reshape(-1, d), K[h], V[h])
        _within(_np(out)[:, 2 * h:2 * h + 2].reshape(-1, d), want, bound, h)
    p.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("batch,capacity,prefix", [(2, 200, 0), (1, 3000, 0), (3, 100, 300), (140, 90, 0)])
def test_step_probabilities(batch, capacity, prefix, d):
    """One workgroup per unit, several, a prefix besides, workgroups of four wavefronts."""
    import torch

    import paper_2502_11147_amd as raas

    say("case precision step %d %d %d %d" % (batch, capacity, prefix, d))
    Hq, Hkv, n = 8, 2, capacity - 1
    rng = np.random.default_rng(capacity)
    (k, K), (v, V) = _data(rng, (batch, Hkv, n, d)), _data(rng, (batch, Hkv, n, d))
    (q, Q), (kn, KN), (vn, VN) = _data(rng, (batch, Hq, d)), _data(rng, (batch, Hkv, d)), _data(rng, (batch, Hkv, d))
    c = raas.WeightCache(batch, 1, Hq, Hkv, d, capacity, 10, "bf16")
    c.prefill(0, k, v)
    p = PK = PV = None
    if prefix:
        (pk, PK), (pv, PV) = _data(rng, (Hkv, prefix, d)), _data(rng, (Hkv, prefix, d))
        p = raas.SharedPrefix(1, Hq, Hkv, d, prefix, batch, "bf16")
        p.store(0, pk, pv)
    out = torch.empty_like(q)
    c.decode_step(0, q, kn, vn, out, prefix=p)
    G = Hq // Hkv
    for b in range(batch):
        for h in range(Hkv):
            keys, values = [K[b, h], KN[b, h][None]], [V[b, h], VN[b, h][None]]
            if prefix:
                keys, values = keys + [PK[h]], values + [PV[h]]
            want, bound = _attention(Q[b, h * G:(h + 1) * G], np.concatenate(keys), np.concatenate(values))
            _within(_np(out)[b, h * G:(h + 1) * G], want, bound, (b, h))
    c.close()


def _prompt(Q, K, lse):
    """(weights, relative error allowed) of one unit: Q [rows][G][d], K [n][d], lse [rows][G] or None.

    For inputs whose products are exact, so that a logit is rounded only at the
    distance from its row's maximum, Y at most (base 2): a probability is off by
    ln 2 * 2 u Y for that, as much for the factor log2(e) / sqrt(d), a few u for
    exponentials and the inverse, n u for the sum it is divided by, doubled where
    numerator and sum have it both; then rows * G of them are added.
    With a prefix that factor's rounding no longer cancels: the logits are off by
    a common delta x, |delta| <= u, and the prefix's sum is not, so that of p_j =
    exp(x_j (1 + delta)) / (sum exp(x (1 + delta)) + exp(lse)) the logarithm moves
    by delta (x_j - sum_j a_j x_j), with sum_j a_j <= 1: by u max |x| at most,
    as any logit held in fp32 does."""
    rows, G, d = Q.shape
    n = len(K)
    w, Y, X = np.zeros(n), 0.0, 0.0
    for i in range(rows):
        last = n - rows + i + 1
        x = Q[i] @ K[:last].T / np.sqrt(d)
        m = x.max(axis=1)
        if lse is not None:
            m = np.maximum(m, lse[i])
        e = np.exp(x - m[:, None])
        z = e.sum(axis=1)
        if lse is not None:
            z = z + np.exp(lse[i] - m)
            X = max(X, np.abs(x).max())
        w[:last] += (e / z[:, None]).sum(axis=0)
        Y = max(Y, (m[:, None] - x).max() / np.log(2.0))
    return w, (4 * np.log(2.0) * Y + n + rows * G + 32 + X) * ref.U32


@pytest.mark.parametrize("prefixed", [False, True])
@pytest.mark.parametrize("dtype,Hq,Hkv,d,n,W", [("f32", 2, 2, 64, 60, 1), ("bf16", 2, 1, 64, 90, 5), ("bf16", 6, 2, 128, 100, 1),
                                                ("f32", 4, 2, 128, 200, 3), ("bf16", 4, 4, 128, 150, 150), ("bf16", 2, 1, 64, 600, 2)])
def test_prompt_weights_of_far_logits(dtype, Hq, Hkv, d, n, W, prefixed):
    """Logits some 2000 or 2900 from 0 and a few apart (integers, so that products are exact)."""
    import torch

    import paper_2502_11147_amd as raas

    say("case precision prompt %s %d %d %d %s" % (dtype, d, n, W, prefixed))
    rng = np.random.default_rng(n + W)
    Q = 16.0 + rng.integers(-1, 2, (1, W, Hq, d))
    K = 16.0 + rng.integers(-1, 2, (1, Hkv, n, d))
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k = (torch.from_numpy(x).to(dt).cuda() for x in (Q, K))
    lse = lse64 = None
    if prefixed:
        lse = (256.0 * np.sqrt(d) + 10.0 + 3.0 * rng.standard_normal((1, W, Hq))).astype(np.float32)
        lse64, lse = lse.astype(np.float64), torch.from_numpy(lse).cuda()
    w = torch.zeros(1, Hkv, n, device="cuda")
    raas.prompt_weights(q, k, w, prefix_lse=lse)
    G = Hq // Hkv
    for h in range(Hkv):
        heads = slice(h * G, (h + 1) * G)
        want, rel = _prompt(Q[0, :, heads], K[0, h], None if lse64 is None else lse64[0, :, heads])
        _within(_np(w)[0, h], want, rel * want + 1e-37, h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_equal_logits_at_the_limit(sign, dtype):
    """Logits of +-4e8, all equal (their products are exact): even weights, the values' mean.

    n + 64 roundings of the sums, and of the mean's type; a log-sum-exp moves by
    a few roundings at its size."""
    import torch

    import paper_2502_11147_amd as raas

    say("case precision limit %s %g" % (dtype, sign))
    rng = np.random.default_rng(5)
    Hq, Hkv, d, n = 4, 2, 64, 300
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    const = lambda c, *shape: torch.full(shape, c, dtype=dt, device="cuda")  # noqa: E731
    x = sign * 8192.0 * 6144.0 * d / np.sqrt(d)
    v = torch.from_numpy(rng.standard_normal((Hkv, n, d)).astype(np.float32)).to(dt).cuda()
    V = _np(v)

    def mean(got, V, what):
        want, A = V.mean(axis=0), np.abs(V).mean(axis=0)
        bound = (len(V) + 64) * ref.U32 * A
        if dtype == "bf16":
            bound = bound + 2.0 ** -15 * A
            bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
        _within(got, np.broadcast_to(want, got.shape), bound, what)

    p = raas.SharedPrefix(1, Hq, Hkv, d, n, 140, dtype)
    p.store(0, const(sign * 6144.0, Hkv, n, d), v)
    for rows in (3, 12, 40, 70, 140):
        out, lse = const(9.0, rows, Hq, d), torch.zeros(rows, Hq, device="cuda")
        p.attend(0, const(8192.0, rows, Hq, d), out, lse)
        for h in range(Hkv):
            mean(_np(out)[:, 2 * h:2 * h + 2].reshape(-1, d), V[h], (rows, h))
        assert np.abs(_np(lse) - x).max() <= 8 * ref.U32 * abs(x)
    w = torch.zeros(1, Hkv, n, device="cuda")
    raas.prompt_weights(const(8192.0, 1, n, Hq, d), const(sign * 6144.0, 1, Hkv, n, d), w)
    want = np.array([sum(2.0 / (i + 1) for i in range(j, n)) for j in range(n)])
    _within(_np(w)[0], np.broadcast_to(want, (Hkv, n)), (n + 2 * n + 64) * ref.U32 * want, "weights")
    c = raas.WeightCache(1, 1, Hq, Hkv, d, n, 8, dtype)
    c.prefill(0, const(sign * 6144.0, 1, Hkv, n - 1, d), v[None, :, 1:].contiguous())
    out, w = const(9.0, 1, Hq, d), torch.zeros(1, Hkv, n, device="cuda")
    c.decode_step(0, const(8192.0, 1, Hq, d), const(sign * 6144.0, 1, Hkv, d), v[None, :, 0].contiguous(), out, weights=w)
    for h in range(Hkv):
        mean(_np(out)[0, 2 * h:2 * h + 2], V[h], ("step", h))
    _within(_np(w)[0], np.full((Hkv, n), 2.0 / n), np.full((Hkv, n), (n + 64) * ref.U32 * 2.0 / n), "step weights")
