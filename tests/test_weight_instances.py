"""Every kernel instance that the launch rules of the weight cache, the shared
prefix and the prompt weights can pick, against the fp64 statements
(tests/weight_reference.py); that the list of the step's is complete (no GPU)."""
from __future__ import annotations

import ctypes
import os

import numpy as np
import pytest

import weight_reference as ref
from harness import say

TYPES = [(t, d) for t in ("bf16", "f32") for d in (64, 128)]

# (wavefronts, workgroups of a unit, whether a kernel of its own ends the step):
# batch, query heads, KV heads, capacity, tokens of the prompts, prefix
STEPS = {
    (4, "fused", False): (129, 8, 2, 70, 66, 0),
    (4, "split", False): (513, 1, 1, 6000, 30, 0),
    (4, "split", True): (513, 2, 1, 8191, 20, 40),
    (8, "fused", False): (3, 14, 2, 101, 90, 33),
    (8, "one", False): (200, 15, 1, 2048, 40, 0),
    (8, "one", True): (200, 14, 1, 2985, 25, 0),
    (8, "split", False): (2, 8, 2, 2100, 500, 50),
    (8, "split", True): (2, 28, 2, 2985, 1000, 0),
}


def _lib():
    import paper_2502_11147_amd as raas

    if not os.path.exists(raas.LIB_PATH):
        from paper_2502_11147_amd import build as b

        b.build()
    return raas.load_library()


class _Plan(ctypes.Structure):  # raas::WeightPlan
    _fields_ = [("waves", ctypes.c_int), ("nsplit", ctypes.c_int), ("fused", ctypes.c_bool), ("finish_parts", ctypes.c_int)]


def _step_kind(units, G, d, capacity, dtype):
    plan = _lib()._ZN4raas16plan_weight_stepEiiiib
    plan.restype, plan.argtypes = _Plan, [ctypes.c_int] * 4 + [ctypes.c_bool]
    p = plan(units, G, d, capacity, dtype == "bf16")
    return p.waves, "fused" if p.fused else "split" if p.nsplit > 1 else "one", p.finish_parts > 0


@pytest.mark.parametrize("dtype,d", TYPES)
def test_every_kind_of_step_is_listed(dtype, d):
    for kind, (batch, Hq, Hkv, C, _, _) in STEPS.items():
        assert _step_kind(batch * Hkv, Hq // Hkv, d, C, dtype) == kind
    for G in range(1, 17):
        for C in (2, 16, 64, 100, 159, 256, 500, 1024, 1500, 2048, 2985, 3943, 6000, 8192, 12000, 30000, 200000, 1 << 20):
            for U in (1, 2, 4, 8, 31, 32, 64, 100, 128, 200, 256, 257, 320, 400, 512, 513, 700, 1024, 2048, 10000, 1000000):
                assert _step_kind(U, G, d, C, dtype) in STEPS, (U, G, C)


# Whether a unit of bf16 at head_dim 128 is split, on both sides of the rule: it
# is where that was measured to be faster
@pytest.mark.parametrize("units,G,capacity,split", [
    (8, 4, 1024, False), (8, 4, 2048, True), (32, 4, 1024, False), (32, 4, 2048, True), (64, 4, 1400, False),
    (128, 4, 1024, False), (128, 4, 2048, False), (128, 7, 3201, False), (152, 4, 4963, False), (656, 4, 2760, False),
    (8, 16, 900, False), (8, 7, 1024, False), (8, 1, 2048, True), (32, 4, 8201, True)])
def test_split_rule(units, G, capacity, split):
    assert (_step_kind(units, G, 128, capacity, "bf16")[1] == "split") == split


def _torch():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("kind", list(STEPS), ids=lambda k: "%d-%s%s" % (k[0], k[1], "-finish" if k[2] else ""))
def test_step(kind, dtype, d):
    """Short prompts, and one sequence whose cache is full, with both kinds of loads."""
    torch = _torch()
    from test_weight_cache import Run, _data

    batch, Hq, Hkv, C, P, prefix = STEPS[kind]
    say("case weight instance %s %s %d" % (kind, dtype, d))
    r = Run(batch, Hq, Hkv, d, C, C // 3, dtype, seed=C + d, prefix=prefix)
    r.prefill([P - i % 7 for i in range(batch)], np.exp(r.rng.standard_normal((batch, Hkv, P))) / P)
    b = batch // 2
    (k, K), (v, V), w = _data(r.rng, (Hkv, C, d), dtype), _data(r.rng, (Hkv, C, d), dtype), np.exp(r.rng.standard_normal((Hkv, C))) / C
    full = [torch.zeros((batch,) + x.shape, dtype=x.dtype, device="cuda") for x in (k, v, torch.from_numpy(w).float())]
    for x, y in zip(full, (k, v, torch.from_numpy(w).float())):
        x[b] = y
    r.cache.prefill(0, full[0], full[1], weights=full[2], mask=[i == b for i in range(batch)])
    for h in range(Hkv):
        r.units[b * Hkv + h].start(K[h], V[h], w[h].astype(np.float32))
    count = _lib()._ZN4raas14count_streamedEiy
    count.restype, count.argtypes = ctypes.c_ulonglong, [ctypes.c_int, ctypes.c_ulonglong]
    evictions = 0
    for t in range(4):
        if t % 2 == 1:  # as if others had pushed the layer out of the memory-side cache
            count(torch.cuda.current_device(), 1 << 40)
        evictions += r.step()
    assert evictions >= 4 * Hkv
    r.check_state()
    r.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_rows_at_head_dim_128(dtype):
    """Both sides of every limit between the prefix kernels, and numbers of parts."""
    torch = _torch()
    import paper_2502_11147_amd as raas
    from test_weight_cache import _data, _np, _within

    G, d, Hkv, most = 2, 128, 2, 260
    rng = np.random.default_rng(12)
    for n in (5, 1300):
        say("case prefix instance %s %d" % (dtype, n))
        p = raas.SharedPrefix(1, G * Hkv, Hkv, d, n, most, dtype)
        (k, K), (v, V) = (_data(rng, (Hkv, n, d), dtype) for _ in range(2))
        p.store(0, k, v)
        q, Q = _data(rng, (most, G * Hkv, d), dtype)
        want = []
        for h in range(Hkv):
            o = ref.prefix_attention(Q[:, h * G:(h + 1) * G].reshape(-1, d), K[h], V[h], dtype == "bf16")
            want.append([y.reshape((most, G) + y.shape[1:]) for y in o])
        o, bound, lse, lb = (np.concatenate(x, axis=1) for x in zip(*want))
        for rows in (1, 8, 9, 32, 33, 64, 65, 128, 129, 192, 193, 260):
            out = torch.full((rows, G * Hkv, d), 9.0, dtype=q.dtype, device="cuda")
            got = torch.full((rows, G * Hkv), 9.0, device="cuda")
            p.attend(0, q[:rows], out, got)
            _within(_np(out), o[:rows], bound[:rows], (n, rows))
            _within(_np(got), lse[:rows], lb[:rows], (n, rows))
        p.close()


# lengths, query heads, KV heads, window: one tile of 16 rows, several shared by
# the workgroup's wavefronts, tiles of their own (rows = window * group)
PROMPTS = [([500, 3], 4, 1, 4), ([300, 20], 4, 1, 6), ([300, 20, 77], 14, 2, 4), ([300, 20], 4, 1, 9), ([200], 6, 1, 4),
           ([200, 41], 16, 1, 4), ([400, 130], 16, 2, 17)]


@pytest.mark.gpu
@pytest.mark.parametrize("prefixed", [False, True])
@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("case", PROMPTS, ids=["%d-%d-%d" % (c[1], c[2], c[3]) for c in PROMPTS])
def test_prompt_windows(case, dtype, d, prefixed):
    torch = _torch()
    import paper_2502_11147_amd as raas
    from test_weight_cache import _data, _np, _within

    lens, Hq, Hkv, W = case
    say("case prompt instance %s %s %d %s" % (case, dtype, d, prefixed))
    B, P, G = len(lens), max(lens), Hq // Hkv
    rng = np.random.default_rng(P + W)
    (q, Q), (k, K) = _data(rng, (B, W, Hq, d), dtype), _data(rng, (B, Hkv, P, d), dtype)
    lse = lse64 = None
    if prefixed:
        lse64 = (3.0 + 2.0 * rng.standard_normal((B, W, Hq))).astype(np.float32)
        lse, lse64 = torch.from_numpy(lse64).cuda(), lse64.astype(np.float64)
    w = torch.full((B, Hkv, P), -3.0, device="cuda")
    raas.prompt_weights(q, k, w, lens=lens, prefix_lse=lse)
    for b in range(B):
        n, rows = lens[b], min(lens[b], W)
        assert (w[b, :, n:] == -3.0).all()
        for h in range(Hkv):
            heads = slice(h * G, (h + 1) * G)
            want, bound = ref.prompt_weights(Q[b, :rows, heads], K[b, h, :n], None if lse is None else lse64[b, :rows, heads])
            _within(_np(w)[b, h, :n], want, bound, (b, h))
