"""The kernels of the quantised cache's steps and of attention of few rows: both kinds of
loads, wavefronts of 0 to 10 and of more than 64 blocks, parts joined with a prefix's."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest

import quant_reference as ref
from test_quant_cache import BITS, _dev, _dtype, _ints, _needs_gpu, _np, _same, _within  # noqa: F401  (a fixture)

gpu = pytest.mark.gpu
BLOCK, WAVES, TARGET, LEAST, WHOLE, MOST_PARTS = 32, 4, 256, 4, 20, 64


def _cut(blocks, hkv):
    """How the kernel of few rows cuts sequences of so many blocks: parts of each and blocks of a part."""
    chunk = -(-sum(blocks) * hkv // TARGET)
    out = []
    for n in blocks:
        each = max(chunk, 8 if n > 16 * LEAST else LEAST)
        parts = 1 if n <= WHOLE else min(MOST_PARTS, -(-n // each))
        out.append((parts, -(-n // parts)))
    return out


def _turns(blocks, hkv):
    """Numbers of blocks that wavefronts take."""
    seen = set()
    for n, (parts, per) in zip(blocks, _cut(blocks, hkv)):
        for p in range(parts):
            lo, hi = min(n, p * per), min(n, (p + 1) * per)
            seen |= {max(0, -(-(hi - lo - w) // WAVES)) for w in range(WAVES)}
    return seen


class Held:
    """Sequences whose whole pages are drawn from a few common ones; their last two pages are their own."""

    def __init__(self, lens, hq, hkv, d, bits, dtype, page, common, seed, missing=0):
        import paper_2502_11147_amd as raas

        rng = self.rng = np.random.default_rng(seed)
        self.lens, self.hq, self.hkv, self.d, self.dt, self.page = lens, hq, hkv, d, _dtype(dtype), page
        self.bits, self.bf16, B = bits, dtype == "bf16", len(lens)
        n, width = common + 2 * B, max(lens) // page + 2
        self.cache = raas.QuantCache(1, hq, hkv, d, n_pages=n, page_size=page, max_batch=B, max_queries=16 // (hq // hkv),
                                     key_bits=bits[0], value_bits=bits[1], dtype=dtype)
        names = rng.permutation(n)
        self.common = self._write(names[None, :common], [0], [common * page])
        self.pages = np.full((B, width), -1)
        for b, m in enumerate(lens):
            full = m // page
            self.pages[b, :full] = names[rng.integers(0, common, full)]
            self.pages[b, full:full + 2] = names[common + 2 * b:common + 2 * b + 2]
        self.own = self._write(self.pages, [m // page * page for m in lens], [m % page for m in lens])
        self.place = {p: i for i, p in enumerate(names[:common])}
        for b in range(missing):  # also the last page, and so the place of a step's token
            full = lens[b] // page
            self.pages[b, full if b % 4 == 3 else rng.integers(0, full + 1)] = [-1, n, -2 ** 31, 2 ** 31 - 1][b % 4]
        self.table = _ints(self.pages)
        self.n = _ints(lens)

    def data(self, *shape):
        x = self.rng.standard_normal(shape).astype(np.float32)
        x[..., ::29] *= 5
        t = _dev(x, self.dt)
        return t, _np(t)

    def _write(self, pages, start, counts):
        shape = (len(pages), self.hkv, max(max(counts), 1), self.d)
        (k, kn), (v, vn) = self.data(*shape), self.data(*shape)
        self.cache.write(0, k, v, _ints(pages), _ints(start), _ints(counts))
        return ref.held(kn, self.bits[0]), ref.held(vn, self.bits[1])

    def tokens(self, b, h, which, new=None):
        """Keys (which 0) or values that sequence b can see, with a step's new token; which tokens those are."""
        page, full, m = self.page, self.lens[b] // self.page, self.lens[b]
        rows, seen = [], []
        for i, p in enumerate(self.pages[b, :full + 1]):
            count = page if i < full else m % page + (new is not None)
            seen += [0 <= p < self.cache.n_pages] * count
            if i < full:
                at = self.place.get(p, 0) * page
                rows.append(self.common[which][0, h, at:at + page])
            else:
                rows.append(self.own[which][b, h, :m % page])
        if new is not None:
            rows.append(new[b, h][None])
        return np.concatenate(rows)[np.array(seen, bool)], np.array(seen, bool)

    def stream(self):
        """The next call finds its layer pushed out of the memory-side cache."""
        import torch

        count = self.cache.lib._ZN4raas14count_streamedEiy
        count.restype, count.argtypes = ctypes.c_ulonglong, [ctypes.c_int, ctypes.c_ulonglong]
        count(torch.cuda.current_device(), 1 << 40)

    def both(self, call, *outs):
        """call() with ordinary loads twice (the first call of a layer may be either) and with
        non-temporal ones: the same bits; the outputs."""
        import torch

        got = []
        for streamed in (False, False, True, True):
            if streamed:
                self.stream()
            for o in outs:
                o.fill_(9.0)
            call()
            got.append([o.clone() for o in outs])
        for x in got[2:]:
            for o, p in zip(x, got[1]):
                assert torch.equal(o, p)
        return [_np(o) for o in got[-1]]

    def check(self, queries, some, prefix=None):
        """A call of `queries` (0: a step) for all sequences; those of `some` against the statement."""
        import torch

        B, G, step = len(self.lens), self.hq // self.hkv, queries == 0
        n = max(queries, 1)
        q, qn = self.data(B, n, self.hq, self.d)
        empty = lambda *shape, dt=self.dt: torch.zeros(*shape, dtype=dt, device="cuda")
        out, lse = empty(B, n, self.hq, self.d), empty(B, n, self.hq, dt=torch.float32)
        kn = vn = None
        if step:
            (k, kn), (v, vn) = self.data(B, self.hkv, self.d), self.data(B, self.hkv, self.d)
            kn, vn = ref.held(kn, self.bits[0]), ref.held(vn, self.bits[1])
            kh, vh = empty(B, self.hkv, self.d), empty(B, self.hkv, self.d)
            args = self.cache.prepare_step(0, q[:, 0], k, v, out[:, 0], self.table, self.n, lse[:, 0], kh, vh,
                                           prefix=None if prefix is None else prefix[0])
            got, gl, gk, gv = self.both(lambda: self.cache.decode_prepared(args), out, lse, kh, vh)
        else:
            got, gl = self.both(lambda: self.cache.attend(0, q, out, self.table, self.n, None, lse), out, lse)
        assert np.isfinite(got).all()
        for b in some:
            for h in range(self.hkv):
                K, seen = self.tokens(b, h, 0, kn)
                V, _ = self.tokens(b, h, 1, vn)
                if step:
                    placed = seen[-1]
                    _same(gk[b, h], kn[b, h] if placed else np.full(self.d, 9.0), (b, h))
                    _same(gv[b, h], vn[b, h] if placed else np.full(self.d, 9.0), (b, h))
                heads = slice(h * G, (h + 1) * G)
                for i in range(n):
                    last = int(seen[:max(0, len(seen) - n + i + 1)].sum())
                    o, ob, l, lb = ref.attention(qn[b, i, heads], K[:last], V[:last], self.bf16,
                                                 None if prefix is None else (prefix[1][h], prefix[2][h]))
                    _within(got[b, i, heads], o, ob, ("out", b, i, h))
                    _within(gl[b, i, heads], l, lb, ("lse", b, i, h))


KINDS = dict(dtype=["bf16", "f32"], bits=BITS, d=[64, 128])


def _kinds(test):
    for name, values in KINDS.items():
        test = pytest.mark.parametrize(name, values, ids=str)(test)
    return gpu(test)


SHORT = [32 * n + 7 * n % 32 for n in range(46)] * 2 + [32 * n for n in (1, 4, 9, 16, 17, 33)]


def test_short_sequences_take_every_number_of_turns():
    blocks = [-(-n // BLOCK) for n in SHORT + [48000, 47001]]
    assert set(range(11)) <= _turns(blocks, 2)
    assert {1, 2} <= {parts for parts, _ in _cut(blocks, 2)} and _cut(blocks, 2)[-1][0] > 30


@_kinds
def test_short_and_long_turns(dtype, bits, d):
    """Wavefronts of 0 to 10 blocks, with a step's new token or a sequence's end at every place of
    the loop, tables without some pages."""
    lens = SHORT + [48000, 47001]
    x = Held(lens, 8, 2, d, bits, dtype, 64, 40, seed=d + bits[0], missing=44)
    some = list(range(0, len(lens) - 2, 1 if d == 64 else 3)) + [len(lens) - 1]
    x.check(0, some)
    x.check(1, some[::2])
    x.check(4, some[1::3])


@_kinds
def test_more_turns_than_lanes(dtype, bits, d):
    """Wavefronts of 69 and more blocks: their pages are read in two turns."""
    lens = [35200 + 37 * b for b in range(66)]
    assert max(_turns([-(-(n + 1) // BLOCK) for n in lens], 1)) > 66
    x = Held(lens, 4, 1, d, bits, dtype, 256, 8, seed=d + bits[1], missing=20)
    x.check(0, [0, 3, 40])
    x.check(4, [1, 65])


@gpu
@pytest.mark.parametrize("shape", [(4, 1, 64), (16, 1, 128), (14, 2, 64), (6, 2, 128)], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_joined_with_a_prefix(dtype, shape):
    """Steps of sequences in 64, 12 and 1 parts beside a prefix in many or one: more sources than lanes."""
    import paper_2502_11147_amd as raas

    hq, hkv, d = shape
    lens = [20000, 601, 5, 0, 2900]
    x = Held(lens, hq, hkv, d, BITS[hq % 4], dtype, 64, 40, seed=hq)
    plan = x.cache.lib._ZN4raas11plan_prefixEiiib
    plan.restype, plan.argtypes = ctypes.c_int, [ctypes.c_int] * 3 + [ctypes.c_bool]
    parts = _cut([-(-(n + 1) // BLOCK) for n in lens], hkv)
    sources = []
    for tokens in (4000, 300, 1, 0):
        p = raas.SharedPrefix(1, hq, hkv, d, 4000, len(lens), dtype)
        (k, kn), (v, vn) = x.data(hkv, max(tokens, 1), d), x.data(hkv, max(tokens, 1), d)
        p.store(0, k if tokens else None, v if tokens else None)
        sources.append(parts[0][0] + plan(hkv, len(lens) * hq // hkv, tokens, dtype == "bf16"))
        x.check(0, range(len(lens)), (p, kn[:, :tokens], vn[:, :tokens]))
    assert parts[0][0] == 64 and parts[1][0] == 1 and parts[4][0] == 12 and max(sources) > 64, (parts, sources)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("queries", [4, 12])
def test_graphs_that_share_a_cache(queries, dtype):
    """A captured step behind a prefix and a captured attention of a draft, of few rows and of many,
    replayed in turn with eager work in between: lengths, inputs and the prefix as they are then."""
    import torch

    import paper_2502_11147_amd as raas

    lens = [3000, 601, 5, 0, 20000]
    x = Held(lens, 8, 2, 64, (4, 8), dtype, 64, 40, seed=queries)
    c = raas.QuantCache(1, 8, 2, 64, n_pages=x.cache.n_pages, page_size=64, max_batch=5, max_queries=queries, key_bits=4,
                        value_bits=8, dtype=dtype)
    shape = (1, 2, 64 * c.n_pages, 64)
    every = torch.arange(c.n_pages, dtype=torch.int32, device="cuda")[None]
    c.write(0, x.data(*shape)[0], x.data(*shape)[0], every, _ints([0]))
    p = raas.SharedPrefix(1, 8, 2, 64, 900, 5, dtype)
    pk, pv = x.data(2, 900, 64)[0], x.data(2, 900, 64)[0]
    p.store(0, pk, pv)
    q, q1, k, v = (x.data(*s)[0] for s in ((5, queries, 8, 64), (5, 8, 64), (5, 2, 64), (5, 2, 64)))
    new = lambda: (torch.zeros_like(q), torch.zeros_like(q1), torch.zeros(5, queries, 8, device="cuda"),  # noqa: E731
                   torch.zeros(5, 8, device="cuda"))
    n = _ints(lens)

    def step(o):
        c.decode_step(0, q1, k, v, o[1], x.table, n, lse=o[3], prefix=p)

    def draft(o):
        c.attend(0, q, o[0], x.table, n, None, o[2])

    outs = new()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(outs)
        draft(outs)
    torch.cuda.synchronize()
    graphs = []
    for call in (step, draft):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(outs)
        graphs.append(g)
    for t in range(6):
        n.copy_(_ints([3000 + 4 * t, 601 + t, 5 * t, -1 if t % 2 else 33, 20000 + 11 * t]))  # (in pages of their own)
        for y in (q, q1, k, v, pk, pv):
            y.copy_(torch.randn(y.shape, device="cuda"))
        p.store(0, pk, pv)
        for o in outs:
            o.fill_(9.0)
        torch.cuda.synchronize()
        for g in graphs if t % 2 else graphs[::-1]:
            g.replay()
        got = [o.clone() for o in outs]
        want = new()
        for o in want:
            o.fill_(9.0)
        for call in (step, draft) if t % 2 else (draft, step):
            call(want)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert not torch.isnan(b).any() and torch.equal(a, b), t
