"""Tokens that some queries of a call of the quantised cache see and others do not."""
from __future__ import annotations

import numpy as np
import pytest

import quant_reference as ref
from test_quant_cache import BITS, Model, _dev, _ints, _needs_gpu, _np, _within  # noqa: F401  (a fixture)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", BITS, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,queries", [(2, 7), (2, 16), (8, 4), (4, 40), (8, 75)])
def test_nan_of_later_tokens(hq, queries, dtype, bits, d):
    """A NaN or infinity reaches no query before its token: the value's those from it on, in the
    channels of its group; the key's all their channels and the log-sum-exp."""
    import torch

    hkv, lens = 2, [130, queries, 64, 97, 700]
    m = Model([0] * 5, hq, hkv, d, bits, dtype, page=32, width=23, max_queries=queries)
    x = m.rng.standard_normal((2, 5, hkv, 700, d)).astype(np.float32)
    bad = []  # (keys 0 or values 1, sequence, KV head, token, first of the group's channels)
    for b, n in enumerate(lens):
        for h, back in ((0, [1, queries // 2]), (1, [queries])):
            if b == 2 and h == 0:
                bad.append((0, b, h, n - 1 - queries // 3, 0))
                continue
            for i, t in enumerate(back):
                bad.append((1, b, h, max(0, n - t), 32 * ((b + i) % (d // 32))))
    for i, (w, b, h, t, c) in enumerate(bad):
        x[w, b, h, t, c + 5 * i % 32] = [np.nan, np.inf, -np.inf][i % 3]
    k, v = _dev(x[0], m.dt), _dev(x[1], m.dt)
    m.cache.write(0, k, v, m.table, _ints([0] * 5), _ints(lens))
    q, qn = m.query(5, queries)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")
    m.cache.attend(0, q, out, m.table, _ints(lens), None, lse)
    got, gl, G = _np(out), _np(lse), hq // hkv
    K, V = (np.nan_to_num(ref.held(_np(y), w), nan=0.0) for y, w in zip((k, v), bits))
    for b, n in enumerate(lens):
        for h in range(hkv):
            heads = slice(h * G, (h + 1) * G)
            mine = [(w, t, c) for w, bb, hh, t, c in bad if (bb, hh) == (b, h)]
            for i in range(queries):
                last = max(0, n - queries + i + 1)
                nan = np.zeros(d, bool)
                for w, t, c in mine:
                    if t < last:
                        nan[slice(c, c + 32) if w == 1 else slice(None)] = True
                keys = any(w == 0 and t < last for w, t, _ in mine)
                what = (b, h, i)
                assert np.array_equal(np.isnan(got[b, i, heads]), np.broadcast_to(nan, (G, d))), what
                assert np.isnan(gl[b, i, heads]).all() == keys and np.isnan(gl[b, i, heads]).any() == keys, what
                if keys or nan.all():
                    continue
                o, ob, l, lb = ref.attention(qn[b, i, heads], K[b, h, :last], V[b, h, :last], m.bf16, half=queries * G > 16)
                _within(gl[b, i, heads], l, lb, ("lse",) + what)
                _within(got[b, i, heads][:, ~nan], o[:, ~nan], ob[:, ~nan], ("out",) + what)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", BITS, ids=str)
def test_groups_of_zeros(bits, d):
    """Padded or silent tokens read as zeros and leave the other channels' outputs the same bits."""
    import torch

    n, queries = 700, 40
    outs, V = [], None
    for zeros in (False, True):
        m = Model([0, 0], 4, 2, d, bits, page=64, width=11, max_queries=queries, seed=9)
        (k, kn), (v, vn) = m.data(2, 2, n, d), m.data(2, 2, n, d)
        if zeros:
            v[0, :, 0, :32], v[0, 1, 650, :32], v[1, :, 300:, :32] = 0, -0.0, 0
            vn = _np(v)
        m.cache.write(0, k, v, m.table, _ints([0, 0]))
        for b in range(2):
            m.K[b], m.V[b] = ref.held(kn[b], bits[0]), ref.held(vn[b], bits[1])
        m.check_held()
        outs.append(m.attend(queries))
    (a, la), (b, lb) = outs
    assert torch.equal(la, lb) and torch.equal(a[..., 32:], b[..., 32:])
