"""The weight cache, the shared prefix and the prompt weights on the GPU
against their fp64 statements (tests/weight_reference.py)."""
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


def _data(rng, shape, dtype, offset=0):
    """N(0, 1) values as the device tensor holds them, `offset` elements into its memory, and in fp64."""
    import torch

    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dt)
    mem = torch.empty(x.numel() + offset, dtype=dt, device="cuda")
    t = mem[offset:].view(shape)
    t.copy_(x)
    return t, x.double().numpy()


def _np(t):
    return t.detach().double().cpu().numpy()


def _within(got, want, bound, what):
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - bound
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, (what, at, got[at], want[at], bound[at])


class Run:
    """A cache of one layer and the reference of each of its units, stepped together."""

    def __init__(self, batch, q_heads, kv_heads, d, capacity, recent, dtype, seed, prefix=0, offset=0, layers=1, layer=0):
        import torch

        import paper_2502_11147_amd as raas

        self.B, self.Hq, self.Hkv, self.d, self.C, self.dtype = batch, q_heads, kv_heads, d, capacity, dtype
        self.G, self.layer, self.offset = q_heads // kv_heads, layer, offset
        self.rng = np.random.default_rng(seed)
        self.cache = raas.WeightCache(batch, layers, q_heads, kv_heads, d, capacity, recent, dtype)
        self.units = [ref.Unit(self.G, d, capacity, recent, dtype == "bf16") for _ in range(batch * kv_heads)]
        self.prefix = self.prefix_kv = None
        if prefix:
            self.prefix = raas.SharedPrefix(layers, q_heads, kv_heads, d, prefix + 5, batch, dtype)
            (k, K), (v, V) = (_data(self.rng, (kv_heads, prefix, d), dtype, offset) for _ in range(2))
            self.prefix.store(layer, k, v)
            self.prefix_kv = list(zip(K, V))
        dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.out = torch.full((batch, q_heads, d), 9.0, dtype=dt, device="cuda")
        self.positions = torch.full((batch, kv_heads, capacity), -9, dtype=torch.int32, device="cuda")
        self.weights = torch.full((batch, kv_heads, capacity), -9.0, device="cuda")
        self.evicted = torch.full((batch, kv_heads), -9, dtype=torch.int32, device="cuda")

    def prefill(self, lens, weights=None, mask=None):
        import torch

        P = max(lens)
        (k, K), (v, V) = (_data(self.rng, (self.B, self.Hkv, P, self.d), self.dtype, self.offset) for _ in range(2))
        w = None if weights is None else torch.from_numpy(weights.astype(np.float32)).cuda()
        self.cache.prefill(self.layer, k if P else None, v if P else None, lens=lens, weights=w, mask=mask)
        for b in range(self.B):
            if mask is not None and not mask[b]:
                continue
            for h in range(self.Hkv):
                n = lens[b]
                self.units[b * self.Hkv + h].start(K[b, h, :n], V[b, h, :n],
                                                   None if weights is None else weights[b, h, :n].astype(np.float32))

    def step(self, active=None):
        import torch

        B, Hq, Hkv, G, d = self.B, self.Hq, self.Hkv, self.G, self.d
        (q, Q), = [_data(self.rng, (B, Hq, d), self.dtype, self.offset)]
        (k, K), (v, V) = (_data(self.rng, (B, Hkv, d), self.dtype, self.offset) for _ in range(2))
        before = [_np(t) for t in (self.out, self.positions, self.weights, self.evicted)]
        act = None if active is None else torch.tensor(active, dtype=torch.int32, device="cuda")
        if active is not None:  # the others' inputs are not looked at
            for b in range(B):
                if not active[b]:
                    for t in (q, k, v):
                        t[b] = float("nan")
        self.cache.decode_step(self.layer, q, k, v, self.out, self.positions, self.weights, self.evicted, active=act,
                               prefix=self.prefix)
        out, pos, w, ev = (_np(t) for t in (self.out, self.positions, self.weights, self.evicted))
        evictions = 0
        for b in range(B):
            if active is not None and not active[b]:
                for now, old in zip((out, pos, w, ev), before):
                    assert np.array_equal(now[b], old[b])
                continue
            for h in range(Hkv):
                u = self.units[b * Hkv + h]
                r, bound, gone = u.step(Q[b, h * G:(h + 1) * G], K[b, h], V[b, h],
                                        None if self.prefix is None else self.prefix_kv[h], ev[b, h])
                where = "sequence %d head %d token %d" % (b, h, u.clock - 1)
                assert ev[b, h] == gone, where
                evictions += gone >= 0
                assert np.array_equal(pos[b, h], u.pos), where
                _within(out[b, h * G:(h + 1) * G], r, bound, where)
                _within(w[b, h], u.w, u.err, where)
        return evictions

    def check_state(self):
        s = self.cache.export_state(self.layer)
        for i, u in enumerate(self.units):
            assert np.array_equal(s["positions"][i], u.pos) and s["clock"][i] == u.clock
            _within(s["weights"][i].astype(np.float64), u.w, u.err, "unit %d" % i)

    def close(self):
        self.cache.close()
        if self.prefix is not None:
            self.prefix.close()


# batch, query heads, KV heads, head_dim, capacity, recent, type, prompt lengths, steps, prefix, offset
STEPS = [
    (1, 4, 1, 64, 64, 16, "f32", [40], 60, 0, 0),
    (2, 8, 2, 128, 48, 12, "bf16", [48, 30], 40, 0, 0),
    (1, 1, 1, 64, 2, 1, "f32", [0], 12, 0, 0),          # the smallest cache, an empty prompt
    (1, 2, 1, 128, 2, 0, "bf16", [1], 12, 0, 1),        # no window: even the newest may go
    (3, 7, 1, 64, 37, 36, "bf16", [37, 1, 0], 50, 0, 1),  # the window covers all but one; odd sizes, odd addresses
    (2, 16, 1, 128, 95, 20, "f32", [95, 64], 24, 0, 1),  # 16 heads
    (1, 14, 2, 64, 129, 3, "f32", [128], 20, 0, 0),
    (1, 32, 2, 128, 33, 8, "bf16", [32], 24, 0, 0),     # 16 heads; one token past a block
    (1, 4, 1, 128, 1500, 700, "bf16", [1490], 20, 0, 0),  # a unit over several workgroups
    (1, 4, 1, 128, 1500, 700, "bf16", [5], 20, 0, 0),     # most of them with nothing to do
    (2, 12, 2, 64, 1025, 100, "f32", [1024, 300], 16, 0, 1),
    (70, 8, 8, 64, 70, 10, "bf16", [70 - i % 9 for i in range(70)], 6, 0, 0),  # more units than workgroups per round
    (2, 8, 2, 128, 40, 8, "bf16", [40, 17], 24, 33, 1),  # with a prefix
    (5, 14, 2, 64, 50, 8, "f32", [50, 1, 0, 33, 50], 12, 130, 0),
    (1, 4, 1, 128, 1100, 64, "bf16", [1100], 8, 1, 0),
    (9, 32, 4, 128, 64, 8, "bf16", [64] * 9, 8, 500, 0),
    (100, 32, 2, 64, 2048, 100, "bf16", [60 - i % 9 for i in range(100)], 3, 0, 0),  # logits that do not fit LDS
    (1, 4, 1, 64, 9000, 3000, "f32", [8995], 12, 0, 0),   # the end of a step in a kernel of its own
    (2, 16, 1, 128, 4100, 100, "bf16", [4100, 50], 6, 40, 1),
]


@pytest.mark.parametrize("case", STEPS, ids=["-".join(str(x) if not isinstance(x, list) else str(x[0]) for x in c) for c in STEPS])
def test_steps(case):
    B, Hq, Hkv, d, C, recent, dtype, lens, steps, prefix, offset = case
    say("case weight steps %s" % (case,))
    r = Run(B, Hq, Hkv, d, C, recent, dtype, seed=11 * C + steps, prefix=prefix, offset=offset)
    P = max(lens)
    r.prefill(lens, np.exp(r.rng.standard_normal((B, Hkv, P))) / max(P, 1))
    evictions = sum(r.step() for _ in range(steps))
    assert evictions > 0 or max(lens) + steps <= C
    r.check_state()
    r.close()


@pytest.mark.parametrize("dtype,prefix", [("bf16", 0), ("f32", 20)])
def test_active_mask_and_restart(dtype, prefix):
    """Sequences at their own pace, others' inputs NaN; then some start over with new prompts, shorter and longer."""
    say("case weight mask %s" % dtype)
    r = Run(4, 8, 2, 64, 45, 11, dtype, seed=5, prefix=prefix)
    r.prefill([45, 20, 0, 60], np.exp(r.rng.standard_normal((4, 2, 60))))
    for t in range(12):
        r.step(active=[1, t % 2, int(t % 3 == 0), 7])
    r.prefill([3, 44, 90, 46], np.exp(r.rng.standard_normal((4, 2, 90))), mask=[1, 0, 1, 0])
    for t in range(12):
        r.step(active=[1, 1, t % 2, 0])
    r.prefill([0, 0, 0, 0], mask=[0, 1, 0, 1])
    for t in range(3):
        r.step()
    r.check_state()
    r.close()


def _levels(rng, shape, n):
    return rng.integers(0, n, shape).astype(np.float64) / 4.0


@pytest.mark.parametrize("C,recent,lens,levels", [
    (40, 8, [41, 100, 2500], 3), (40, 0, [41, 1024, 1025], 1), (40, 39, [300, 41, 40], 2),
    (1030, 100, [3000, 2048, 1031], 5), (2, 1, [2047, 3, 2], 2), (64, 10, [5000, 70, 64], 100000)])
def test_prefill_keeps_the_heaviest(C, recent, lens, levels):
    """Weights on few levels: of equal ones the newer stay."""
    say("case weight prefill %d %d %s %d" % (C, recent, lens, levels))
    r = Run(3, 4, 2, 64, C, recent, "f32", seed=C + levels)
    w = _levels(r.rng, (3, 2, max(lens)), levels)
    w[0, 0, :3] = -0.0  # equal to 0
    r.prefill(lens, w)
    r.check_state()
    r.step()
    r.prefill(lens)  # no weights: the newest stay
    r.check_state()
    r.close()


def test_prefill_of_many_sequences():
    """More sequences than one launch's lengths."""
    say("case weight many sequences")
    r = Run(600, 1, 1, 64, 8, 2, "bf16", seed=3)
    lens = [i % 12 for i in range(600)]
    r.prefill(lens, _levels(r.rng, (600, 1, 11), 4))
    r.check_state()
    r.step()
    r.prefill(lens[::-1], mask=[i >= 555 for i in range(600)])
    r.check_state()
    r.close()


def test_layers_are_apart():
    r = Run(2, 4, 1, 64, 20, 4, "bf16", seed=8, prefix=9, layers=3, layer=2)
    other = r.cache.export_state(0)
    r.prefill([20, 25], np.exp(r.rng.standard_normal((2, 1, 25))))
    for _ in range(5):
        r.step()
    r.check_state()
    for key, x in r.cache.export_state(0).items():
        assert np.array_equal(x, other[key])
    r.close()


PREFIX = [
    # rows, query heads, KV heads, head_dim, tokens, type, offset
    (1, 1, 1, 64, 1, "f32", 0), (1, 4, 1, 128, 31, "bf16", 1), (3, 14, 2, 64, 33, "f32", 1), (4, 16, 4, 128, 32, "bf16", 0),
    (5, 7, 1, 128, 1000, "bf16", 0), (17, 8, 8, 64, 257, "bf16", 0), (33, 32, 4, 128, 700, "bf16", 1),
    (40, 16, 1, 64, 130, "f32", 0), (64, 32, 2, 128, 515, "f32", 0), (130, 4, 1, 128, 4099, "bf16", 0),
    (2, 4, 2, 128, 9001, "bf16", 0), (300, 8, 1, 64, 70, "bf16", 0),
]


@pytest.mark.parametrize("case", PREFIX, ids=["-".join(map(str, c)) for c in PREFIX])
def test_prefix_attention(case):
    import torch

    import paper_2502_11147_amd as raas

    rows, Hq, Hkv, d, n, dtype, offset = case
    say("case prefix %s" % (case,))
    G = Hq // Hkv
    rng = np.random.default_rng(n)
    p = raas.SharedPrefix(2, Hq, Hkv, d, n + 40, rows + 1, dtype)
    (k2, _), (v2, _) = (_data(rng, (Hkv, n + 40, d), dtype) for _ in range(2))
    p.store(1, k2, v2)  # a longer one first
    (k, K), (v, V) = (_data(rng, (Hkv, n, d), dtype, offset) for _ in range(2))
    p.store(1, k, v)
    q, Q = _data(rng, (rows, Hq, d), dtype, offset)
    out, _ = _data(rng, (rows, Hq, d), dtype, offset)
    lse = torch.full((rows, Hq), 7.0, device="cuda")
    p.attend(1, q, out, lse)
    o, s = _np(out), _np(lse)
    again = torch.empty_like(out)
    p.attend(1, q, again)  # the same bits, without the log-sum-exp
    assert torch.equal(out, again)
    for b in range(rows):
        for h in range(Hkv):
            heads = slice(h * G, (h + 1) * G)
            r, bound, want, lb = ref.prefix_attention(Q[b, heads], K[h], V[h], dtype == "bf16")
            _within(o[b, heads], r, bound, (b, h))
            _within(s[b, heads], want, lb, (b, h))
    p.close()


@pytest.mark.parametrize("dtype,Hkv,n", [("bf16", 1, 2100), ("bf16", 3, 1500), ("f32", 2, 1100)])
def test_prefix_rows_of_one_handle(dtype, Hkv, n):
    """Fewer rows than the handle may take: every tile of rows and number of parts
    fits its scratch."""
    import torch

    import paper_2502_11147_amd as raas

    say("case prefix rows %s %d" % (dtype, Hkv))
    G, d, most = 2, 64, 330
    rng = np.random.default_rng(n)
    p = raas.SharedPrefix(1, G * Hkv, Hkv, d, n, most, dtype)
    (k, K), (v, V) = (_data(rng, (Hkv, n, d), dtype) for _ in range(2))
    p.store(0, k, v)
    q, Q = _data(rng, (most, G * Hkv, d), dtype)
    want = []
    for h in range(Hkv):
        x = Q[:, h * G:(h + 1) * G].reshape(-1, d)
        o, bound, lse, lb = ref.prefix_attention(x, K[h], V[h], dtype == "bf16")
        want.append([y.reshape((most, G) + y.shape[1:]) for y in (o, bound, lse, lb)])
    o, bound, lse, lb = (np.concatenate(x, axis=1) for x in zip(*want))
    for rows in (1, 8, 9, 16, 17, 32, 33, 64, 65, 128, 129, 192, 193, 256, 257, 320, 321, 330):
        out = torch.full((rows, G * Hkv, d), 9.0, dtype=q.dtype, device="cuda")
        got = torch.full((rows, G * Hkv), 9.0, device="cuda")
        p.attend(0, q[:rows], out, got)
        _within(_np(out), o[:rows], bound[:rows], rows)
        _within(_np(got), lse[:rows], lb[:rows], rows)
    p.close()


def test_empty_prefix():
    import torch

    import paper_2502_11147_amd as raas

    p = raas.SharedPrefix(1, 4, 2, 64, 10, 3, "bf16")
    p.store(0, None, None)
    q = torch.randn(3, 4, 64, device="cuda").bfloat16()
    out, lse = torch.full_like(q, 5.0), torch.zeros(3, 4, device="cuda")
    p.attend(0, q, out, lse)
    assert (out == 0).all() and (lse == -float("inf")).all()
    p.attend(0, q[:0], out[:0])
    r = Run(3, 4, 2, 64, 20, 4, "bf16", seed=1)
    r.prefill([20, 4, 0], np.ones((3, 2, 20)))
    r.prefix, r.prefix_kv = p, [(np.zeros((0, 64)), np.zeros((0, 64)))] * 2
    for _ in range(3):
        r.step()
    r.close()


PROMPT = [
    # lengths, query heads, KV heads, head_dim, window, type, offset
    ([1], 1, 1, 64, 1, "f32", 0), ([5, 0, 3], 4, 2, 64, 5, "f32", 1), ([33, 17], 7, 1, 128, 33, "bf16", 1),
    ([300], 4, 1, 128, 300, "bf16", 0), ([700, 255, 64], 8, 4, 64, 20, "bf16", 0), ([130, 129], 16, 1, 128, 130, "f32", 0),
    ([2100, 900], 4, 2, 128, 3, "bf16", 0), ([1111], 14, 2, 64, 1, "f32", 0), ([40, 2, 600], 3, 1, 64, 64, "bf16", 0),
    ([9] * 300, 1, 1, 64, 4, "f32", 0),
    # (more than 16 pieces of the keys, and of the rows)
    ([9001, 5, 4500], 2, 1, 64, 3, "bf16", 0), ([1200, 70], 4, 1, 64, 1200, "bf16", 0), ([5003], 6, 2, 128, 2, "f32", 0),
]


@pytest.mark.parametrize("prefixed", [False, True])
@pytest.mark.parametrize("case", PROMPT, ids=["-".join(map(str, [c[0][0], len(c[0])] + list(c[1:]))) for c in PROMPT])
def test_prompt_weights(case, prefixed):
    import torch

    import paper_2502_11147_amd as raas

    lens, Hq, Hkv, d, W, dtype, offset = case
    say("case prompt weights %s %s" % (case, prefixed))
    B, P, G = len(lens), max(lens), Hq // Hkv
    rng = np.random.default_rng(P + W)
    (q, Q), (k, K) = _data(rng, (B, W, Hq, d), dtype, offset), _data(rng, (B, Hkv, P, d), dtype, offset)
    lse = lse64 = None
    if prefixed:
        lse = torch.from_numpy((3.0 + 2.0 * rng.standard_normal((B, W, Hq))).astype(np.float32)).cuda()
        lse[0, 0, 0] = -float("inf")  # an empty prefix
        lse64 = _np(lse)
    w = torch.full((B, Hkv, P), -3.0, device="cuda")
    raas.prompt_weights(q, k, w, lens=lens, prefix_lse=lse)
    got = _np(w)
    for b in range(B):
        n = lens[b]
        rows = min(n, W)
        assert (got[b, :, n:] == -3.0).all()
        for h in range(Hkv if n else 0):
            heads = slice(h * G, (h + 1) * G)
            want, bound = ref.prompt_weights(Q[b, :rows, heads], K[b, h, :n],
                                             None if lse is None else lse64[b, :rows, heads])
            _within(got[b, h, :n], want, bound, (b, h))
            if lse is None:
                assert abs(got[b, h, :n].sum() - rows * G) <= bound.sum() + 1e-12


def _problem(seed, dtype="bf16"):
    """A shared prompt, private prompts behind it, and the handles that serve them."""
    import torch

    import paper_2502_11147_amd as raas

    rng = np.random.default_rng(seed)
    B, Hq, Hkv, d, S, P, C = 3, 8, 2, 128, 70, 60, 40
    s = dict(B=B, Hq=Hq, Hkv=Hkv, d=d, S=S, P=P, C=C, lens=[60, 33, 7])
    for name, shape in (("sk", (Hkv, S, d)), ("sv", (Hkv, S, d)), ("k", (B, Hkv, P, d)), ("v", (B, Hkv, P, d)),
                        ("q", (B, P, Hq, d))):
        s[name], s[name + "64"] = _data(rng, shape, dtype)
    s["prefix"] = raas.SharedPrefix(1, Hq, Hkv, d, S, B * P, dtype)
    s["cache"] = raas.WeightCache(B, 1, Hq, Hkv, d, C, 10, dtype)
    s["rng"], s["raas"], s["torch"] = rng, raas, torch
    return s


def test_run_together():
    """A shared prompt stored once; each private prompt's weights counted behind it; admission; steps over both."""
    s = _problem(4)
    torch, raas, B, Hq, Hkv, d, P, C = s["torch"], s["raas"], s["B"], s["Hq"], s["Hkv"], s["d"], s["P"], s["C"]
    G = Hq // Hkv
    s["prefix"].store(0, s["sk"], s["sv"])
    rows = s["q"].view(B * P, Hq, d)
    out, lse = torch.empty_like(rows), torch.empty(B * P, Hq, device="cuda")
    s["prefix"].attend(0, rows, out, lse)
    w = torch.zeros(B, Hkv, P, device="cuda")
    raas.prompt_weights(s["q"], s["k"], w, lens=s["lens"], prefix_lse=lse.view(B, P, Hq))
    s["cache"].prefill(0, s["k"], s["v"], lens=s["lens"], weights=w)
    got, lse64 = _np(w), _np(lse).reshape(B, P, Hq)
    units = []
    for b in range(B):
        n = s["lens"][b]
        for h in range(Hkv):
            heads = slice(h * G, (h + 1) * G)
            for i in range(0, n, 7):
                r = ref.prefix_attention(s["q64"][b, i, heads], s["sk64"][h], s["sv64"][h], True)
                _within(lse64[b, i, heads], r[2], r[3], (b, h, i))
            want, bound = ref.prompt_weights(s["q64"][b, :n, heads], s["k64"][b, h, :n], lse64[b, :n, heads])
            _within(got[b, h, :n], want, bound, (b, h))
            u = ref.Unit(G, d, C, 10, True)
            u.start(s["k64"][b, h, :n], s["v64"][b, h, :n], got[b, h, :n])
            units.append(u)
    o = torch.empty(B, Hq, d, dtype=torch.bfloat16, device="cuda")
    pos = torch.empty(B, Hkv, C, dtype=torch.int32, device="cuda")
    ev = torch.empty(B, Hkv, dtype=torch.int32, device="cuda")
    for t in range(30):
        (q, Q), (k, K), (v, V) = (_data(s["rng"], (B, H, d), "bf16") for H in (Hq, Hkv, Hkv))
        s["cache"].decode_step(0, q, k, v, o, pos, evicted=ev, prefix=s["prefix"])
        for i, u in enumerate(units):
            b, h = divmod(i, Hkv)
            r, bound, gone = u.step(Q[b, h * G:(h + 1) * G], K[b, h], V[b, h], (s["sk64"][h], s["sv64"][h]),
                                    int(ev[b, h]))
            assert ev[b, h] == gone and np.array_equal(_np(pos)[b, h], u.pos)
            _within(_np(o)[b, h * G:(h + 1) * G], r, bound, (t, i))


@pytest.mark.parametrize("capacity", [40, 2100])
def test_graph_replays(capacity):
    """A captured step with a prefix, and captured prompt weights, replayed
    between eager steps, against a cache that is stepped eagerly alone: the
    same bits. The cache fills up and the prefix is exchanged between replays."""
    import torch

    import paper_2502_11147_amd as raas

    rng = np.random.default_rng(capacity)
    B, Hq, Hkv, d = 2, 8, 2, 64
    mk = lambda *shape: _data(rng, shape, "bf16")[0]  # noqa: E731
    caches = [raas.WeightCache(B, 1, Hq, Hkv, d, capacity, 6, "bf16") for _ in range(2)]
    prefixes = [raas.SharedPrefix(1, Hq, Hkv, d, 300, B, "bf16") for _ in range(2)]
    k0, v0 = mk(B, Hkv, capacity - 5, d), mk(B, Hkv, capacity - 5, d)
    sk, sv = mk(Hkv, 50, d), mk(Hkv, 50, d)
    w0 = torch.rand(B, Hkv, capacity - 5, device="cuda")
    for c, p in zip(caches, prefixes):
        c.prefill(0, k0, v0, weights=w0)
        p.store(0, sk, sv)
    q, k, v = mk(B, Hq, d), mk(B, Hkv, d), mk(B, Hkv, d)
    shape = (B, Hkv, capacity)
    outs = [(torch.zeros(B, Hq, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(shape, dtype=torch.int32, device="cuda"),
             torch.zeros(shape, device="cuda"), torch.zeros(B, Hkv, dtype=torch.int32, device="cuda")) for _ in range(2)]
    pq, pk = mk(B, 9, Hq, d), mk(B, Hkv, 100, d)
    pw = torch.zeros(B, Hkv, 100, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        caches[1].decode_step(0, q, k, v, *outs[1], prefix=prefixes[1])
        raas.prompt_weights(pq, pk, pw, lens=[100, 41])
    for t in range(14):
        for x in (q, k, v, pq):
            x.copy_(torch.from_numpy(rng.standard_normal(tuple(x.shape)).astype(np.float32)))
        if t == 7:  # a longer prefix
            sk, sv = mk(Hkv, 300, d), mk(Hkv, 300, d)
            for p in prefixes:
                p.store(0, sk, sv)
        caches[0].decode_step(0, q, k, v, *outs[0], prefix=prefixes[0])
        want = torch.zeros_like(pw)
        raas.prompt_weights(pq, pk, want, lens=[100, 41])
        if t % 4 == 3:  # an eager step between the replays
            caches[1].decode_step(0, q, k, v, *outs[1], prefix=prefixes[1])
        else:
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(pw, want), t
        torch.cuda.synchronize()
        same = [torch.equal(a, b) for a, b in zip(*outs)]
        # (a captured step keeps the prefix's split of its capture, which rounds otherwise)
        assert same[1] and same[3] and (t >= 7 or all(same)), (t, same)
        if t >= 7:
            assert (outs[0][0].float() - outs[1][0].float()).abs().max() <= 2.0 ** -6
            assert (outs[0][2] - outs[1][2]).abs().max() <= 1e-5


def test_side_stream():
    """Every call on a stream that is not the current one."""
    import torch

    import paper_2502_11147_amd as raas

    side = torch.cuda.Stream()
    rng = np.random.default_rng(0)
    got = []
    for stream in (None, side):
        rng = np.random.default_rng(0)
        mk = lambda *shape: _data(rng, shape, "f32")[0]  # noqa: E731
        sk, sv, k0, v0 = mk(2, 90, 64), mk(2, 90, 64), mk(3, 2, 50, 64), mk(3, 2, 50, 64)
        qw, q, k, v = mk(3, 50, 4, 64), mk(3, 4, 64), mk(3, 2, 64), mk(3, 2, 64)
        w, out, out2 = torch.zeros(3, 2, 50, device="cuda"), torch.zeros(3, 4, 64, device="cuda"), torch.zeros(3, 4, 64, device="cuda")
        weights = torch.zeros(3, 2, 40, device="cuda")
        torch.cuda.synchronize()
        c = raas.WeightCache(3, 1, 4, 2, 64, 40, 4, "f32", stream=stream)
        p = raas.SharedPrefix(1, 4, 2, 64, 90, 3, "f32", stream=stream)
        p.store(0, sk, sv, stream=stream)
        raas.prompt_weights(qw, k0, w, stream=stream)
        c.prefill(0, k0, v0, weights=w, stream=stream)
        c.decode_step(0, q, k, v, out, weights=weights, prefix=p, stream=stream)
        p.attend(0, q, out2, stream=stream)
        state = c.export_state(0, stream=stream)
        torch.cuda.synchronize()
        got.append([out, out2, weights, w, torch.from_numpy(state["weights"]), torch.from_numpy(state["positions"])])
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_two_streams_at_once():
    """Two caches with a prefix each, stepped on two streams with nothing between
    them, as each alone: the same bits."""
    import torch

    import paper_2502_11147_amd as raas

    say("case weight two streams")
    rng = np.random.default_rng(6)
    B, Hq, Hkv, d, C = 5, 8, 2, 128, 3000
    mk = lambda *shape: _data(rng, shape, "bf16")[0]  # noqa: E731
    data = [[mk(Hkv, 400, d), mk(Hkv, 400, d), mk(B, Hkv, C, d), mk(B, Hkv, C, d), mk(9, B, Hq, d), mk(9, B, Hkv, d),
             mk(9, B, Hkv, d)] for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for together in (False, True):
        torch.cuda.synchronize()
        made = []
        for (sk, sv, k0, v0, _, _, _), s in zip(data, streams):
            p = raas.SharedPrefix(1, Hq, Hkv, d, 400, B, stream=s)
            c = raas.WeightCache(B, 1, Hq, Hkv, d, C, 100, stream=s)
            p.store(0, sk, sv, stream=s)
            c.prefill(0, k0, v0, stream=s)
            made.append((c, p, torch.zeros(9, B, Hq, d, dtype=torch.bfloat16, device="cuda"),
                         torch.zeros(B, Hkv, C, device="cuda")))
        torch.cuda.synchronize()
        order = [(i, t) for t in range(9) for i in range(2)] if together else [(i, t) for i in range(2) for t in range(9)]
        for i, t in order:
            c, p, out, w = made[i]
            c.decode_step(0, data[i][4][t], data[i][5][t], data[i][6][t], out[t], weights=w, prefix=p, stream=streams[i])
            if not together:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        got.append([x for m in made for x in m[2:]])
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_load_kinds_round_alike():
    """A layer that other caches' steps push out of the memory-side cache is read
    with other loads: the same bits."""
    import torch

    import paper_2502_11147_amd as raas

    say("case weight load kinds")
    B, Hq, Hkv, d, C = 32, 16, 8, 128, 2048
    g = torch.Generator(device="cuda").manual_seed(3)
    mk = lambda *shape: torch.randn(*shape, generator=g, device="cuda").bfloat16()  # noqa: E731
    k0, v0, q, k, v = mk(B, Hkv, C, d), mk(B, Hkv, C, d), mk(6, B, Hq, d), mk(6, B, Hkv, d), mk(6, B, Hkv, d)
    caches = [raas.WeightCache(B, 1, Hq, Hkv, d, C, 100) for _ in range(3)]
    for c in caches:
        c.prefill(0, k0, v0)
    outs = [(torch.zeros_like(q), torch.zeros(B, Hkv, C, device="cuda")) for _ in range(2)]
    for t in range(6):  # alone
        caches[0].decode_step(0, q[t], k[t], v[t], outs[0][0][t], weights=outs[0][1])
    for t in range(6):  # with another one's steps in between
        caches[1].decode_step(0, q[t], k[t], v[t], outs[1][0][t], weights=outs[1][1])
        caches[2].decode_step(0, q[t], k[t], v[t], torch.empty_like(q[t]))
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_offsets_past_two_to_the_31():
    """The last unit's rows lie past 2^31 elements in both handles."""
    import torch

    import paper_2502_11147_amd as raas

    C, Hkv, d = 1 << 20, 17, 128
    say("case weight offsets")
    r = Run(1, Hkv, Hkv, d, C, 0, "bf16", seed=2)
    r.prefill([40], np.exp(r.rng.standard_normal((1, Hkv, 40))))
    p = raas.SharedPrefix(1, Hkv, Hkv, d, C, 1, "bf16")
    (k, K), (v, V) = (_data(r.rng, (Hkv, 70, d), "bf16") for _ in range(2))
    p.store(0, k, v)
    r.prefix, r.prefix_kv = p, list(zip(K, V))
    r.step()
    r.step()
    r.close()
