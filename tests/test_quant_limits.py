"""The quantised cache at the ends of what include/raas.h allows: logits far from 0,
the largest calls, what a handle reserves."""
from __future__ import annotations

import ctypes
import math

import numpy as np
import pytest

import quant_reference as ref
from test_quant_cache import BITS, _config, _dev, _dtype, _ints, _needs_gpu, _np, _within, lib  # noqa: F401  (fixtures)

U32 = ref.U32
gpu = pytest.mark.gpu


def _attend(K, V, q, bits, dtype):
    """out, lse [queries][hq], [d] of the last queries, as fp64; what the values are held as."""
    import torch

    import paper_2502_11147_amd as raas

    (hkv, n, d), (queries, hq) = V.shape, q.shape[:2]
    pages = -(-n // 64)
    c = raas.QuantCache(1, hq, hkv, d, n_pages=pages, max_batch=1, max_queries=queries, key_bits=bits[0], value_bits=bits[1],
                        dtype=dtype)
    table = _ints(np.arange(pages)[None, ::-1])
    v = _dev(V[None], _dtype(dtype))
    c.write(0, _dev(K[None], _dtype(dtype)), v, table, _ints([0]))
    qd = _dev(q[None], _dtype(dtype))
    assert np.array_equal(_np(qd)[0], q)
    out, lse = torch.full_like(qd, 9.0), torch.full((1, queries, hq), 9.0, device="cuda")
    c.attend(0, qd, out, table, _ints([n]), None, lse)
    c.close()
    return _np(out)[0], _np(lse)[0], ref.held(_np(v)[0], bits[1])


def _check(got, gl, V, gaps, x, largest, dtype, half, what):
    """gaps [n]: what token j's logit, all of whose sums are exact, lies above x [queries][hq]. Softmax
    does not depend on x: the exponent fma(logit, scale, -m) is a difference of two
    neighbours, rounded once at its own size, and a reference m that is rounded at the
    logits' size moves all probabilities of a row by one factor. So a probability is off
    by (n + 64 + 4 max gap) u of itself, an output as tests/quant_reference.py says
    beyond that; a log-sum-exp moves by a few roundings at its size."""
    queries, hq, d = got.shape
    hkv, n = V.shape[:2]
    for i in range(queries):
        last = n - queries + i + 1
        e = np.exp(gaps[:last] - gaps[:last].max())
        a = e / e.sum()
        rel = (last + 64 + 4 * np.ptp(gaps[:last]) + (0 if dtype == "bf16" else 2 * last)) * U32
        log = x[i] + gaps[:last].max() + math.log(e.sum())
        assert (np.abs(gl[i] - log) <= 8 * U32 * np.abs(largest) + rel).all(), (what, i, gl[i], log)
        for h in range(hkv):
            want, A = a @ V[h, :last], a @ np.abs(V[h, :last])
            bound = rel * A
            if dtype == "bf16":
                bound = bound + (2.0 ** -11 * A + 2.0 ** -32 * a.max() * np.abs(V[h, :last]).sum(0) if half else 2.0 ** -15 * A)
                bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
            heads = slice(h * hq // hkv, (h + 1) * hq // hkv)
            _within(got[i, heads], np.broadcast_to(want, got[i, heads].shape), np.broadcast_to(bound, got[i, heads].shape),
                    what + (i, h))


def _queries(rng, x, d, queries, hq):
    """Constants, one a row, that keys of 6144 turn into logits up to x; their logits."""
    c = x * rng.uniform(0.9, 1.0, (queries, hq, 1)) / (6144.0 * math.sqrt(d))
    unit = 2.0 ** np.floor(np.log2(c) - 7)
    c = np.floor(c / unit) * unit  # bf16
    return c, (c * 6144.0 * d / math.sqrt(d))[..., 0]


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", BITS, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("queries", [1, 6, 40])
def test_equal_logits_far_out(queries, dtype, bits, d):
    """All tokens' logits equal, up to +-4.99e8: even weights, the values' mean, up to values of
    2^75 (2^72 times normal numbers) and far below 1."""
    rng = np.random.default_rng(queries + d + bits[0])
    hkv, n = 2, 300
    hq = 4
    for x in (1e5, 3e6, 2e7, 6e7, 1.2e8, 2.08e8, 3e8, 4.2e8, 4.99e8):
        for sign in (1.0, -1.0):
            for size in (1.0, 2.0 ** 72, 2.0 ** -60):
                c, logit = _queries(rng, x, d, queries, hq)
                V = rng.standard_normal((hkv, n, d)) * size
                got, gl, held = _attend(np.full((hkv, n, d), sign * 6144.0), V, np.broadcast_to(c, (queries, hq, d)), bits, dtype)
                _check(got, gl, held, np.zeros(n), sign * logit, x, dtype, queries * hq // hkv > 16, (x, sign, size))


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", BITS, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("queries", [1, 40])
def test_rising_logits_far_out(queries, dtype, bits, d):
    """Logits that rise from block to block by a few units (a channel of small queries:
    every sum is a multiple of 32 below 2^29, thus exact), while all lie far from 0."""
    rng = np.random.default_rng(queries + d + bits[1])
    hkv, hq, n = 2, 4, 300
    steps = np.array([0, 1, 2, 3, 4, 6, 8, 12])  # times 512: the 4-bit grid beside 6144
    at = steps[np.minimum(np.arange(n) // 32, 7)]
    for x in (1e5, 2e6, 1e7, 2.5e7, 4e7):
        for sign in (1.0, -1.0):
            c, _ = _queries(rng, x, d, queries, hq)
            q = np.repeat(c, d, axis=2)
            q[..., 0] = 2.0 ** -4
            K = np.full((hkv, n, d), sign * 6144.0)
            K[..., 0] = 512.0 * at
            V = rng.standard_normal((hkv, n, d))
            got, gl, held = _attend(K, V, q, bits, dtype)
            logit = sign * (c * 6144.0 * (d - 1) / math.sqrt(d))[..., 0]
            _check(got, gl, held, 32.0 * at / math.sqrt(d), logit, x, dtype, queries * hq // hkv > 16, (x, sign))


@pytest.mark.parametrize("units,refused", [(4096 * 2048, False), (4096 * 2049, True), (4096 * 4096, True)])
def test_units_of_a_call(lib, units, refused):  # noqa: F811
    """max_batch * n_kv_heads workgroups and those of cut sequences, of 256 threads, are within 2^32."""
    import paper_2502_11147_amd as raas

    heads = units // 4096
    cfg = _config(n_layers=1, n_q_heads=heads, n_kv_heads=heads, head_dim=64, page_size=32, n_pages=1, max_batch=4096,
                  max_queries=1)
    h = ctypes.c_void_p()
    code = lib.raas_create_quant_cache(ctypes.byref(cfg), None, ctypes.byref(h))
    assert (code == raas.E_INVALID) == refused  # (without a GPU a call in range fails otherwise)
    if refused:
        assert b"max_batch * n_kv_heads" in lib.raas_last_error()
    lib.raas_destroy_quant_cache(h)


@gpu
def test_the_most_units():
    """4096 sequences of 2048 KV heads, all behind one page."""
    import torch

    import paper_2502_11147_amd as raas

    B, H, d, n = 4096, 2048, 64, 31
    rng = np.random.default_rng(1)
    c = raas.QuantCache(1, H, H, d, n_pages=1, page_size=32, max_batch=B)
    k, v = (_dev(rng.standard_normal((1, H, n, d)).astype(np.float32), torch.bfloat16) for _ in range(2))
    c.write(0, k, v, _ints([[0]]), _ints([0]))
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(B, 1, H, d, generator=g, device="cuda", dtype=torch.bfloat16)
    out, lse = torch.full_like(q, 9.0), torch.full((B, 1, H), 9.0, device="cuda")
    c.attend(0, q, out, torch.zeros(B, 1, dtype=torch.int32, device="cuda"), _ints([n] * B), None, lse)
    K, V = ref.held(_np(k)[0], 4), ref.held(_np(v)[0], 4)
    b = np.concatenate([[0, B - 1, 0, B - 1], rng.integers(0, B, 300)])
    h = np.concatenate([[0, H - 1, H - 1, 0], rng.integers(0, H, 300)])
    at = torch.from_numpy(b).cuda(), 0, torch.from_numpy(h).cuda()
    got, gl, qn = _np(out[at]), _np(lse[at]), _np(q[at])
    for i in range(len(b)):
        o, ob, l, lb = ref.attention(qn[i][None], K[h[i]], V[h[i]], True)
        _within(got[i][None], o, ob, ("out", b[i], h[i]))
        _within(gl[i][None], l, lb, ("lse", b[i], h[i]))
    assert not (lse == 9.0).any()
    c.close()


class _Scratch(ctypes.Structure):  # raas::QuantScratch
    _fields_ = [("rows", ctypes.c_size_t), ("arrivals", ctypes.c_size_t)]


def _scratch(lib, batch, queries, hkv, G):  # noqa: F811
    f = lib._ZN4raas13quant_scratchEiiii
    f.restype, f.argtypes = _Scratch, [ctypes.c_int] * 4
    x = f(batch, queries, hkv, G)
    return x.rows, x.arrivals


def test_scratch_is_that_of_the_calls_that_can_be(lib):  # noqa: F811
    """Rows of parts: 2 * 256 slots of 16 rows for up to 16 rows per KV head, 2 * 1024 of 32 beyond,
    64 per tile if that is less."""
    for batch, queries, hkv, G, rows in ((128, 1, 8, 4, 512 * 16), (128, 4, 8, 4, 512 * 16), (1, 16, 2, 1, 128 * 16),
                                         (128, 5, 8, 4, 2048 * 32), (1, 17, 2, 1, 128 * 32), (1, 40, 2, 1, 256 * 32),
                                         (4096, 1, 2048, 1, 512 * 16)):
        assert _scratch(lib, batch, queries, hkv, G) == (rows, batch * hkv)


@gpu
@pytest.mark.parametrize("queries", [1, 20])
@pytest.mark.parametrize("pages", [40, 9000])
def test_tokens_never_written(pages, queries):
    """A new cache's tokens are zeros, also where another's lay before: NaN in every page of it."""
    import torch

    import paper_2502_11147_amd as raas

    make = lambda: raas.QuantCache(2, 4, 2, 128, n_pages=pages, page_size=256, max_batch=1, max_queries=20,  # noqa: E731
                                   key_bits=8, value_bits=4)
    n = min(pages, 4096) * 256
    nan = torch.full((1, 2, n, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    table = torch.arange(pages - n // 256, pages, dtype=torch.int32, device="cuda")[None]
    c = make()
    for layer in range(2):
        c.write(layer, nan, nan, table, _ints([0]))
    torch.cuda.synchronize()
    c.close()
    c = make()
    out = torch.full((1, queries, 4, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((1, queries, 4), 9.0, device="cuda")
    for layer in range(2):
        k, v = torch.full_like(nan, 9.0), torch.full_like(nan, 9.0)
        c.read(layer, k, v, table, _ints([0]))
        assert not k.any() and not v.any()
        c.attend(layer, torch.randn_like(out), out, table, _ints([n]), None, lse)
        assert not out.any()
        want = np.log(n - queries + 1.0 + np.arange(queries))
        assert np.abs(_np(lse)[0] - want[:, None]).max() <= (n + 64) * U32 + 8 * U32 * want.max()
    c.close()


@gpu
def test_first_call_on_another_stream():
    """A new cache is ready for every stream: clearing 9 GB does not reach into what is written at once."""
    import torch

    import paper_2502_11147_amd as raas

    n = 140000
    rng = np.random.default_rng(3)
    k, v = (_dev(rng.standard_normal((1, 4, 256, 128)).astype(np.float32), torch.bfloat16) for _ in range(2))
    table, start = _ints([[n - 1, n // 2, n - 2, 0]]), _ints([0])
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        c = raas.QuantCache(1, 4, 4, 128, n_pages=n, page_size=64, max_batch=1, key_bits=8, value_bits=8)
        c.write(0, k, v, table, start, stream=s)
        torch.cuda.synchronize()
        c.read(0, ko, vo, table, start)
        assert np.array_equal(_np(ko), ref.held(_np(k), 8)) and np.array_equal(_np(vo), ref.held(_np(v), 8))
        c.close()
