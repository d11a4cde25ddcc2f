"""Calls of the operators around a cache that evicts by accumulated attention
weight, each through the public entry points of the package:

  step      one decode step of such a cache (WeightCache.decode_prepared): the
            lightest token outside the recent window gives its place to the
            new one, attention over the held tokens, and every held token's
            weight grows by its softmax probabilities, summed over the heads
  admit     new requests (WeightCache.prefill keeps the heaviest prompt tokens)
            and their first step
  prefix    attention of every sequence's queries over one prompt that the
            batch shares (SharedPrefix.attend)
  together  a step whose sequences attend to the shared prompt besides
            (prepare_step(prefix=...))
  weights   the weights that a prompt's own queries give its tokens
            (prompt_weights): column sums of the causal softmax over the last
            `window` queries

A case is a dict of plain values:
  kind      one of the five
  batch, q_heads, kv_heads, head_dim, dtype
            the layer
  capacity, recent
            tokens held per sequence and KV head, and how many of the newest
            are never evicted
  prompt    prompt tokens per sequence; with ragged, the longest
  ragged    prompt lengths spread over 3/4 prompt .. prompt, and about a
            quarter of the sequences sits out each step (the active mask)
  prefix    tokens of the shared prompt
  window    queries per sequence of `weights`

Inputs are N(0, 1) queries, keys and values from the seed; a query leans
towards one earlier key, as the queries of a reasoning stream do, so that
weights concentrate. Weights that a prompt brings along spread over a few
powers of e around those of one query. The steps' inputs form a ring.
"""
from __future__ import annotations

import math
import random

import torch

own = False

RING = 31

_LLAMA = dict(q_heads=32, kv_heads=8, head_dim=128)
_QWEN = dict(q_heads=28, kv_heads=4, head_dim=128)
_BASE = dict(dtype="bf16", capacity=0, recent=0, prompt=0, ragged=False, prefix=0, window=0)

# limits of a drawn case: K and V bytes of a cache or a prompt, multiply-adds
# of a prefix or a prompt's weights, all within the largest listed ones
MOST_CACHE_BYTES = 128 * 8 * 8192 * 128 * 2 * 2
MOST_PREFIX_MACS = 128 * 32 * 32768 * 128 * 2
MOST_WEIGHT_PAIRS = 32 * 4096 * 4096


def _case(name, kind, **kw):
    c = dict(_BASE, name=name, kind=kind)
    c.update(kw)
    return c


def listed():
    return [
        # the smallest cache: one unit in fp32, where a step is one chain of latencies
        _case("step-f32-d64-b1-C256", "step", batch=1, q_heads=4, kv_heads=1, head_dim=64, dtype="f32", capacity=256,
              recent=64, prompt=256),
        # one user at a Llama-3.1-8B-shaped layer: latency again, eight units
        _case("step-llama-b1-C1024", "step", batch=1, **_LLAMA, capacity=1024, recent=512, prompt=1024),
        # four users with long caches of an odd size: a unit over many workgroups
        _case("step-llama-b4-C8201", "step", batch=4, **_LLAMA, capacity=8201, recent=1024, prompt=8201),
        # the serving load that the benchmark quotes, 32 users with 2048 tokens each
        _case("step-llama-b32-C2048", "step", batch=32, **_LLAMA, capacity=2048, recent=1024, prompt=2048),
        # the largest: 128 users with 8192 tokens each
        _case("step-llama-b128-C8192", "step", batch=128, **_LLAMA, capacity=8192, recent=2048, prompt=8192),
        # 32 requests admitted with ragged prompts of up to 4000 tokens, half of which stay
        _case("admit-llama-b32-P4000-C2048", "admit", batch=32, **_LLAMA, capacity=2048, recent=512, prompt=4000,
              ragged=True),
        # 32 samples of one question with few-shot examples
        _case("prefix-llama-b32-P4096", "prefix", batch=32, **_LLAMA, prefix=4096),
        # 128 samples over one long document
        _case("prefix-llama-b128-P32768", "prefix", batch=128, **_LLAMA, prefix=32768),
        # a small fp32 layer, seven samples, an odd prompt
        _case("prefix-f32-d64-b7-P1001", "prefix", batch=7, q_heads=14, kv_heads=2, head_dim=64, dtype="f32",
              prefix=1001),
        # 64 samples of one 8192-token prompt at their own pace, 1024 tokens of its own each
        _case("together-llama-b64-C1024-P8192", "together", batch=64, **_LLAMA, capacity=1024, recent=256, prompt=1000,
              ragged=True, prefix=8192),
        # a whole prompt's weights, every query counted
        _case("weights-llama-b1-P4096", "weights", batch=1, **_LLAMA, prompt=4096, window=4096),
        # ragged prompts, the last 64 queries of each
        _case("weights-qwen-b8-P8191-W64", "weights", batch=8, **_QWEN, prompt=8191, window=64, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        c = dict(_BASE)
        c["kind"] = rng.choice(["step", "step", "admit", "prefix", "prefix", "together", "weights"])
        shape = rng.choice([(32, 8, 128), (32, 8, 128), (28, 4, 128), (16, 4, 128), (4, 1, 64), (14, 2, 64), (8, 8, 128),
                            (32, 2, 128)])
        c["q_heads"], c["kv_heads"], c["head_dim"] = shape
        c["dtype"] = "f32" if rng.random() < (0.5 if shape[2] == 64 else 0.15) else "bf16"
        c["batch"] = _log_int(rng, 1, 128)
        c["ragged"] = c["kind"] != "prefix" and rng.random() < 0.3
        if c["kind"] in ("step", "admit", "together"):
            c["capacity"] = _log_int(rng, 128, 8192)
            c["recent"] = int(c["capacity"] * rng.uniform(0.05, 0.9))
            over = rng.uniform(1.0, 2.5) if c["kind"] == "admit" else rng.uniform(0.5, 1.2)
            c["prompt"] = int(c["capacity"] * over)
        if c["kind"] in ("prefix", "together"):
            c["prefix"] = _log_int(rng, 256, 32768)
        if c["kind"] == "weights":
            c["batch"] = _log_int(rng, 1, 32)
            c["prompt"] = _log_int(rng, 64, 16384)
            c["window"] = c["prompt"] if rng.random() < 0.3 else min(c["prompt"], _log_int(rng, 1, 256))
        # fp32 layers up to an eighth of the largest
        heavy = 8 if c["dtype"] == "f32" else 1
        cache = c["batch"] * c["kv_heads"] * max(c["capacity"], c["prompt"]) * c["head_dim"] * 2 * _esz(c)
        macs = c["batch"] * c["q_heads"] * c["prefix"] * c["head_dim"] * 2
        pairs = c["batch"] * c["q_heads"] * c["window"] * c["prompt"]
        if cache * heavy <= MOST_CACHE_BYTES and macs * heavy <= MOST_PREFIX_MACS and pairs * heavy <= MOST_WEIGHT_PAIRS:
            return c


def _esz(c):
    return 2 if c["dtype"] == "bf16" else 4


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _lens(c, seed):
    """Prompt length of every sequence."""
    if not c["ragged"]:
        return [c["prompt"]] * c["batch"]
    r = random.Random(seed * 7919 + 1)
    return [r.randint(c["prompt"] * 3 // 4, c["prompt"]) for _ in range(c["batch"])]


def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _inputs(c, seed):
    """Every input of the case, by name."""
    device = _device()
    g = torch.Generator(device=device).manual_seed(seed)
    B, Hq, Hkv, d, dt = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], _dtype(c)
    P, S = c["prompt"], c["prefix"]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=device)

    def lean(q, k):
        """q [..., G, d] towards the keys k [..., d]."""
        return q + 3.0 * (k / k.norm(dim=-1, keepdim=True)).unsqueeze(-2)

    x = {}
    if S:
        x["prefix_k"], x["prefix_v"] = randn(Hkv, S, d).to(dt), randn(Hkv, S, d).to(dt)
    if P:
        x["prompt_k"] = randn(B, Hkv, P, d).to(dt)
    if c["kind"] == "weights":
        W = c["window"]
        at = torch.randint(0, max(1, P * 3 // 4 - W + 1), (B, W, Hkv), generator=g, device=device)
        k = x["prompt_k"].float()[torch.arange(B, device=device)[:, None, None], torch.arange(Hkv, device=device), at]
        x["q"] = lean(randn(B, W, Hkv, Hq // Hkv, d), k).reshape(B, W, Hq, d).to(dt)
        return x
    if P:
        x["prompt_v"] = randn(B, Hkv, P, d).to(dt)
        x["prompt_w"] = torch.exp(2.0 * randn(B, Hkv, P)) * (Hq / Hkv / P)
        k = x["prompt_k"][:, :, torch.randint(0, P, (RING,), generator=g, device=device)].permute(2, 0, 1, 3).float()
    else:
        k = x["prefix_k"][:, torch.randint(0, S, (RING,), generator=g, device=device)].transpose(0, 1).unsqueeze(1).float()
    x["q"] = lean(randn(RING, B, Hkv, Hq // Hkv, d), k).reshape(RING, B, Hq, d).to(dt)
    x["k"], x["v"] = randn(RING, B, Hkv, d).to(dt), randn(RING, B, Hkv, d).to(dt)
    x["active"] = (torch.rand(RING, B, generator=g, device=device) < (0.75 if c["ragged"] else 2.0)).to(torch.int32)
    return x


class _State:
    pass


def prepare(case, seed):
    c, x = case, _inputs(case, seed)
    s = _State()
    s.case, s.x, s.lens, s.pos = c, x, _lens(c, seed), 0
    s.masked = c["ragged"] and c["kind"] != "admit"
    B, Hq, Hkv, d, C = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["capacity"]

    def zeros(*shape, dtype=torch.int32):
        return torch.zeros(*shape, dtype=dtype, device=_device())

    if c["kind"] == "weights":
        s.out = {"weights": zeros(B, Hkv, c["prompt"], dtype=torch.float32)}
    elif c["kind"] == "prefix":
        s.out = {"out": zeros(B, Hq, d, dtype=_dtype(c)), "lse": zeros(B, Hq, dtype=torch.float32)}
    else:
        s.out = {"out": zeros(B, Hq, d, dtype=_dtype(c)), "positions": zeros(B, Hkv, C),
                 "weights": zeros(B, Hkv, C, dtype=torch.float32), "evicted": zeros(B, Hkv)}
    s.prefix = s.cache = None
    if own:
        import paper_2502_11147_amd as raas

        s.raas = raas
        if c["prefix"]:
            s.prefix = raas.SharedPrefix(1, Hq, Hkv, d, max_tokens=c["prefix"], max_rows=B, dtype=c["dtype"])
            s.prefix.store(0, x["prefix_k"], x["prefix_v"])
        if C:
            s.cache = raas.WeightCache(B, 1, Hq, Hkv, d, capacity=C, recent=c["recent"], dtype=c["dtype"])
            s.args = [s.cache.prepare_step(0, x["q"][i], x["k"][i], x["v"][i], s.out["out"], s.out["positions"],
                                           s.out["weights"], s.out["evicted"], prefix=s.prefix,
                                           active=x["active"][i] if s.masked else None) for i in range(RING)]
            if c["kind"] != "admit":
                s.cache.prefill(0, x["prompt_k"], x["prompt_v"], lens=s.lens, weights=x["prompt_w"])
    else:
        s.len = torch.tensor(s.lens, device=_device())
        if C and c["kind"] != "admit":
            _plain_prefill(s)
    if c["kind"] in ("step", "together"):  # held in the cache from here on
        for name in ("prompt_k", "prompt_v", "prompt_w"):
            del x[name]
    return s


def run(state):
    s = state
    kind, x, i = s.case["kind"], s.x, s.pos
    s.pos = (i + 1) % RING
    if not own:
        if kind == "weights":
            return _plain_weights(s)
        if kind == "prefix":
            return _plain_prefix(s, x["q"][i])
        if kind == "admit":
            _plain_prefill(s)
        return _plain_step(s, x["q"][i], x["k"][i], x["v"][i], x["active"][i] if s.masked else None)
    if kind == "weights":
        s.raas.prompt_weights(x["q"], x["prompt_k"], s.out["weights"], lens=s.lens)
    elif kind == "prefix":
        s.prefix.attend(0, x["q"][i], s.out["out"], s.out["lse"])
    else:
        if kind == "admit":
            s.cache.prefill(0, x["prompt_k"], x["prompt_v"], lens=s.lens, weights=x["prompt_w"])
        s.cache.decode_prepared(s.args[i])
    return s.out


# ---------------------------------------------------------------------------
# The plain forms: elementary torch operations in 32 bits.

def _plain_weights(s):
    """w_j = sum over queries i >= j and the group's heads of softmax_j(q_i k_j / sqrt(d))."""
    c, q, k = s.case, s.x["q"].float(), s.x["prompt_k"].float()
    B, W, P, Hkv, d = c["batch"], c["window"], c["prompt"], c["kv_heads"], c["head_dim"]
    G = c["q_heads"] // Hkv
    q = q.reshape(B, W, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B * Hkv, G * W, d)
    x = torch.bmm(q, k.reshape(B * Hkv, P, d).transpose(1, 2).contiguous()).reshape(B, Hkv, G, W, P) / math.sqrt(d)
    row, col = torch.arange(W, device=q.device), torch.arange(P, device=q.device)
    count = s.len.clamp(max=W)
    at = (s.len - count)[:, None] + row
    sees = (col <= at[:, :, None]) & (row < count[:, None])[:, :, None]
    x.masked_fill_(~sees[:, None, None], -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True).clamp(min=-1e30))
    x /= x.sum(-1, keepdim=True).clamp(min=1e-30)
    held = col < s.len[:, None]
    s.out["weights"] = torch.where(held[:, None], x.sum((2, 3)), s.out["weights"])
    return s.out


def _prefix_logits(s, q):
    """[Hkv, B*G, S] scaled logits of the queries q [B, Hq, d] over the shared prompt."""
    c = s.case
    B, Hkv, d = c["batch"], c["kv_heads"], c["head_dim"]
    q = q.float().reshape(B, Hkv, -1, d).transpose(0, 1).reshape(Hkv, -1, d)
    return torch.bmm(q, s.x["prefix_k"].float().transpose(1, 2).contiguous()) / math.sqrt(d)


def _plain_prefix(s, q):
    c = s.case
    B, Hkv, d = c["batch"], c["kv_heads"], c["head_dim"]
    x = _prefix_logits(s, q)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - m)
    z = p.sum(-1, keepdim=True)
    out = torch.bmm(p, s.x["prefix_v"].float()) / z
    s.out["out"] = out.reshape(Hkv, B, -1, d).transpose(0, 1).reshape(B, -1, d).to(_dtype(c))
    s.out["lse"] = (m + torch.log(z)).reshape(Hkv, B, -1).transpose(0, 1).reshape(B, -1).contiguous()
    return s.out


def _plain_prefill(s):
    """Keeps every token of a prompt that fits, else the `recent` newest and the heaviest others (of equal ones the later)."""
    c, x = s.case, s.x
    B, Hkv, d, C, P = c["batch"], c["kv_heads"], c["head_dim"], c["capacity"], c["prompt"]
    U = B * Hkv
    n = s.len.repeat_interleave(Hkv)[:, None]
    at = torch.arange(P, device=n.device)
    w = x["prompt_w"].reshape(U, P)
    rank = torch.where(at >= n - c["recent"], torch.full_like(w, math.inf), w)
    rank = torch.where(at < n, rank, torch.full_like(w, -math.inf))
    rank = torch.cat([torch.full((U, max(0, C - P)), -math.inf, device=n.device), rank], 1)
    kept = rank.shape[1] - 1 - torch.sort(rank.flip(1), dim=1, descending=True, stable=True).indices[:, :C] - max(0, C - P)
    held = (kept >= 0) & (kept < n)
    kept = torch.sort(torch.where(held, kept, torch.full_like(kept, P)), 1).values
    held = kept < P
    idx = kept.clamp(max=P - 1)
    s.position = torch.where(held, kept, torch.full_like(kept, -1))
    s.weight = torch.where(held, w.gather(1, idx), torch.zeros_like(w[:, :1]))
    rows = idx[..., None].expand(U, C, d)
    s.K = x["prompt_k"].reshape(U, P, d).gather(1, rows)
    s.V = x["prompt_v"].reshape(U, P, d).gather(1, rows)
    s.clock = n[:, 0].clone()
    s.unit = torch.arange(U, device=n.device)


def _plain_step(s, q, k, v, active):
    c, u, C = s.case, s.unit, s.case["capacity"]
    B, Hkv, d = c["batch"], c["kv_heads"], c["head_dim"]
    U, G = B * Hkv, c["q_heads"] // Hkv
    on = torch.ones_like(u, dtype=torch.bool) if active is None else active.bool().repeat_interleave(Hkv)
    # the place: the first free one, else the lightest token's outside the window (of equal ones the oldest's)
    free = s.position < 0
    full = ~free.any(1)
    old = (s.position < s.clock[:, None] - c["recent"]) & ~free
    w = s.weight.masked_fill(~old, math.inf)
    tie = old & (w == w.amin(1, keepdim=True))
    victim = torch.where(tie, s.position, torch.iinfo(torch.int64).max).argmin(1)
    place = torch.where(full, victim, free.int().argmax(1))
    evicted = torch.where(full, s.position[u, victim], -1)
    s.K[u, place] = torch.where(on[:, None], k.reshape(U, d), s.K[u, place])
    s.V[u, place] = torch.where(on[:, None], v.reshape(U, d), s.V[u, place])
    s.position[u, place] = torch.where(on, s.clock, s.position[u, place])
    s.weight[u, place] = torch.where(on, 0.0, s.weight[u, place])
    held = s.position >= 0
    # attention, over the shared prompt besides
    qf = q.float().reshape(U, G, d)
    x = torch.bmm(qf, s.K.float().transpose(1, 2).contiguous()) / math.sqrt(d)
    x = x.masked_fill(~held[:, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    if c["prefix"]:
        xp = _prefix_logits(s, q)
        m = torch.maximum(m, xp.amax(-1).reshape(Hkv, B, G).transpose(0, 1).reshape(U, G, 1))
    p = torch.exp(x - m)
    z, out = p.sum(-1, keepdim=True), torch.bmm(p, s.V.float())
    if c["prefix"]:
        pp = torch.exp(xp - m.reshape(B, Hkv, G).transpose(0, 1).reshape(Hkv, B * G, 1))
        z = z + pp.sum(-1).reshape(Hkv, B, G).transpose(0, 1).reshape(U, G, 1)
        out = out + torch.bmm(pp, s.x["prefix_v"].float()).reshape(Hkv, B, G, d).transpose(0, 1).reshape(U, G, d)
    s.weight = torch.where(on[:, None], s.weight + (p / z).sum(1), s.weight)
    s.clock = s.clock + on
    o = s.out
    rows = on.reshape(B, Hkv)[:, :1]
    o["out"] = torch.where(rows[..., None], (out / z).reshape(B, Hkv * G, d).to(_dtype(c)), o["out"])
    o["positions"] = torch.where(rows[..., None], s.position.reshape(B, Hkv, C).int(), o["positions"])
    o["weights"] = torch.where(rows[..., None], s.weight.reshape(B, Hkv, C), o["weights"])
    o["evicted"] = torch.where(rows, evicted.reshape(B, Hkv).int(), o["evicted"])
    return o


# ---------------------------------------------------------------------------
# The definition in 64 bits, sequence by sequence and head by head.

def exact(case, seed):
    c, x, lens = case, _inputs(case, seed), _lens(case, seed)
    B, Hq, Hkv, d, C = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["capacity"]
    G, scale = Hq // Hkv, 1.0 / math.sqrt(d)
    dev = x["q"].device
    f64 = dict(dtype=torch.float64, device=dev)
    if c["kind"] == "weights":
        got = torch.zeros(B, Hkv, c["prompt"], **f64)
        for b in range(B):
            n = lens[b]
            rows = min(n, c["window"])
            for h in range(Hkv):
                keys = x["prompt_k"][b, h, :n].double()
                for r0 in range(0, rows, 1024):
                    r1 = min(rows, r0 + 1024)
                    q = x["q"][b, r0:r1, h * G:(h + 1) * G].double()
                    a = torch.matmul(q.reshape(-1, d), keys.t().contiguous()).reshape(r1 - r0, G, n) * scale
                    last = n - rows + torch.arange(r0, r1, device=dev)
                    hidden = torch.arange(n, device=dev)[None] > last[:, None]
                    got[b, h, :n] += torch.softmax(a.masked_fill(hidden[:, None], -math.inf), 2).sum((0, 1))
        return {"weights": got}
    q, k, v = (x[name][0].double() for name in ("q", "k", "v"))
    pk = x["prefix_k"].double() if c["prefix"] else None
    pv = x["prefix_v"].double() if c["prefix"] else None
    if c["kind"] == "prefix":
        out, lse = torch.empty(B, Hq, d, **f64), torch.empty(B, Hq, **f64)
        for h in range(Hkv):
            heads = slice(h * G, (h + 1) * G)
            a = torch.matmul(q[:, heads].reshape(-1, d), pk[h].t().contiguous()) * scale
            lse[:, heads] = torch.logsumexp(a, 1).reshape(B, G)
            out[:, heads] = torch.matmul(torch.softmax(a, 1), pv[h]).reshape(B, G, d)
        return {"out": out, "lse": lse}
    r = {"out": torch.zeros(B, Hq, d, **f64), "weights": torch.zeros(B, Hkv, C, **f64),
         "positions": torch.zeros(B, Hkv, C, dtype=torch.int32, device=dev),
         "evicted": torch.zeros(B, Hkv, dtype=torch.int32, device=dev)}
    active = x["active"][0].tolist() if c["ragged"] and c["kind"] != "admit" else [1] * B
    for b in range(B):
        if not active[b]:
            continue
        n, age = lens[b], torch.arange(lens[b], device=dev)
        for h in range(Hkv):
            w0 = x["prompt_w"][b, h, :n]
            kept = age
            if n > C:
                first = n - c["recent"]
                order = torch.sort(w0[:first], stable=True).indices  # lightest first, of equal ones the oldest
                kept = torch.cat([torch.sort(order[n - C:]).values, age[first:]])
            pos, w = torch.full((C,), -1, dtype=torch.int64, device=dev), torch.zeros(C, **f64)
            m = len(kept)
            pos[:m], w[:m] = kept, w0[kept].double()
            place, evicted = m, -1
            if m == C:
                old = torch.nonzero(pos < n - c["recent"])[:, 0]
                at = old[torch.sort(w[old], stable=True).indices[0]]  # places are in the order of positions here
                place, evicted = int(at), int(pos[at])
            keys, vals = torch.zeros(C, d, **f64), torch.zeros(C, d, **f64)
            keys[:m], vals[:m] = x["prompt_k"][b, h, kept].double(), x["prompt_v"][b, h, kept].double()
            pos[place], w[place], keys[place], vals[place] = n, 0.0, k[b, h], v[b, h]
            m = max(m, place + 1)
            if pk is not None:
                keys, vals = torch.cat([keys[:m], pk[h]]), torch.cat([vals[:m], pv[h]])
            else:
                keys, vals = keys[:m], vals[:m]
            a = torch.softmax(torch.matmul(q[b, h * G:(h + 1) * G], keys.t().contiguous()) * scale, 1)
            r["out"][b, h * G:(h + 1) * G] = torch.matmul(a, vals)
            w[:m] += a.sum(0)[:m]
            r["weights"][b, h], r["positions"][b, h], r["evicted"][b, h] = w, pos.int(), evicted
    return r


def work(case):
    """One pass. A step reads keys, values, positions and weights of the held
    tokens, writes the weights, and both state outputs; an admission reads and
    writes the kept tokens' keys and values once besides, and every prompt
    weight. A prefix is read once whatever the batch; a prompt's weights need
    its keys once and one product, the shared causal part left out."""
    c = case
    e, d, G = _esz(c), c["head_dim"], c["q_heads"] // c["kv_heads"]
    B, Hkv, Hq, C = c["batch"], c["kv_heads"], c["q_heads"], c["capacity"]
    lens = _lens(c, 0)
    if c["kind"] == "weights":
        b = f = 0.0
        for n in lens:
            rows = min(n, c["window"])
            pairs = rows * n - rows * (rows - 1) / 2.0
            b += Hkv * n * (d * e + 4) + rows * Hq * d * e
            f += 2.0 * pairs * Hq * d
        return {"bytes": b, "flops": f}
    b = 2.0 * Hkv * c["prefix"] * d * e
    share = 0.75 if c["ragged"] and c["kind"] != "admit" else 1.0
    f = 4.0 * B * share * Hq * c["prefix"] * d
    if c["kind"] == "prefix":
        return {"bytes": b + 2.0 * B * Hq * d * e + 4.0 * B * Hq, "flops": f}
    for n in lens:
        held = min(C, n + 1)
        b += share * (Hkv * (held * (2.0 * d * e + 12) + 8 * C + 4 * d * e) + 2 * Hq * d * e)
        f += share * 4.0 * held * Hq * d
        if c["kind"] == "admit":
            b += Hkv * (4 * n + min(C, n) * (4.0 * d * e + 8))
    return {"bytes": b, "flops": f}
