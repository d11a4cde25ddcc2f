"""Calls of the operators around a paged cache that holds keys and values in 4
or 8 bits, each through the public entry points of the package:

  store  new tokens of every sequence are quantised as they are written
         (QuantCache.write) and read back as values (QuantCache.read)
  read   held tokens read back as values
  step   one decode step (QuantCache.decode_prepared): the new token is
         quantised and stored, every query head attends to all held tokens,
         and to a prompt that the batch shares, if there is one
  chunk  several new tokens a sequence, a piece of a prompt or a draft: written
         (QuantCache.write), then their queries attend causally to everything
         held (QuantCache.attend)

A group of 32 channels of a token shares a power of two X, the least with
max |x| < 7 X for 4 bits (e2m1, values up to 6) and < 464 X for 8 (e4m3, up to
448): the largest value and half its step. Every value is the nearest multiple
that the type has, of two equally near the one with the even code.

A case is a dict of plain values:
  kind       one of the four
  batch, q_heads, kv_heads, head_dim, dtype
             the layer
  key_bits, value_bits, page
             the cache: bits of a value, tokens of a page
  held       tokens that a sequence holds before the call; with ragged, the most
  new        tokens that a sequence brings (`read`: reads); with ragged, the most
  ragged     held tokens spread over 3/4 held .. held, new ones over half of new
             .. new, and about a quarter of the sequences sits out
  prefix     tokens of the shared prompt

Keys are N(0, 1) with four channels of each head six times as large, as rotary
keys have; values are N(0, 1); a query leans towards one held key. The pages of
a sequence lie scattered over the cache.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_LLAMA = dict(q_heads=32, kv_heads=8, head_dim=128)
_QWEN = dict(q_heads=28, kv_heads=4, head_dim=128)
_BASE = dict(dtype="bf16", key_bits=4, value_bits=4, page=64, held=0, new=1, ragged=False, prefix=0)

# limits of a drawn case: values of a cache, values written and read back,
# pairs of a query head and a token, all within the largest listed ones
MOST_CACHE = 128 * 8 * 8192 * 128
MOST_COPIED = 32 * 8 * 4000 * 128
MOST_PAIRS = 4 * 32 * 512 * 16384


def _case(name, kind, **kw):
    c = dict(_BASE, name=name, kind=kind)
    c.update(kw)
    return c


def listed():
    return [
        # the smallest cache: one unit in fp32 and 8 bits, where a step is one chain of latencies
        _case("step-f32-d64-b1-n200-k8v8", "step", batch=1, q_heads=4, kv_heads=1, head_dim=64, dtype="f32", key_bits=8,
              value_bits=8, page=32, held=200),
        # one user at a Llama-3.1-8B-shaped layer
        _case("step-llama-b1-n1000-k4v4", "step", batch=1, **_LLAMA, held=1000),
        # 32 users at their own pace behind a shared prompt, 8 bits
        _case("step-llama-b32-n4096-k8v8-P2048", "step", batch=32, **_LLAMA, key_bits=8, value_bits=8, held=4096,
              ragged=True, prefix=2048),
        # the largest: 128 users with 8192 tokens each in 4 bits
        _case("step-llama-b128-n8192-k4v4", "step", batch=128, **_LLAMA, held=8192),
        # three long documents, keys in 8 bits beside values in 4
        _case("step-qwen-b3-n60001-k8v4", "step", batch=3, **_QWEN, key_bits=8, page=128, held=60001),
        # a draft of four tokens behind the last one, for 16 users
        _case("chunk-llama-b16-n5-L4000-k4v4", "chunk", batch=16, **_LLAMA, held=4000, new=5, ragged=True),
        # a whole prompt in one piece
        _case("chunk-llama-b1-n4096-k8v8", "chunk", batch=1, **_LLAMA, key_bits=8, value_bits=8, new=4096),
        # pieces of 512 tokens of four long prompts
        _case("chunk-llama-b4-n512-L15872-k4v4", "chunk", batch=4, **_LLAMA, held=15872, new=512),
        # 32 requests admitted with ragged prompts
        _case("store-llama-b32-P4000-k4v4", "store", batch=32, **_LLAMA, new=4000, ragged=True),
        # a few tokens behind an odd number of held ones, a small fp32 layer
        _case("store-f32-d64-b2-P77-k8v4", "store", batch=2, q_heads=14, kv_heads=2, head_dim=64, dtype="f32", key_bits=8,
              page=32, held=45, new=77),
        # eight sequences leave for another cache
        _case("read-llama-b8-n8192-k4v4", "read", batch=8, **_LLAMA, held=8192, new=8192),
        # part of one sequence, from an odd token on
        _case("read-qwen-b1-n1000-k8v8", "read", batch=1, **_QWEN, key_bits=8, value_bits=8, page=32, held=1333, new=1000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        c = dict(_BASE)
        c["kind"] = rng.choice(["step", "step", "chunk", "chunk", "store", "read"])
        shape = rng.choice([(32, 8, 128), (32, 8, 128), (28, 4, 128), (16, 4, 128), (4, 1, 64), (14, 2, 64), (8, 8, 128),
                            (32, 2, 128)])
        c["q_heads"], c["kv_heads"], c["head_dim"] = shape
        c["dtype"] = "f32" if rng.random() < (0.5 if shape[2] == 64 else 0.15) else "bf16"
        c["key_bits"], c["value_bits"] = rng.choice([(4, 4), (4, 4), (8, 8), (8, 4), (4, 8)])
        c["page"] = rng.choice([32, 64, 128, 256])
        c["batch"] = _log_int(rng, 1, 128)
        c["ragged"] = rng.random() < 0.4
        if c["kind"] == "step":
            c["held"] = _log_int(rng, 64, 65536)
            c["prefix"] = _log_int(rng, 256, 16384) if rng.random() < 0.25 else 0
        elif c["kind"] == "chunk":
            c["batch"] = _log_int(rng, 1, 32)
            c["new"] = _log_int(rng, 2, 16) if rng.random() < 0.4 else _log_int(rng, 17, 4096)
            c["held"] = 0 if rng.random() < 0.25 else _log_int(rng, 64, 32768)
        else:
            c["new"] = _log_int(rng, 1, 16384)
            c["held"] = c["new"] + rng.randint(0, 500) if c["kind"] == "read" else rng.randint(0, 500)
        # fp32 layers up to an eighth of the largest
        heavy = 8 if c["dtype"] == "f32" else 1
        rows = c["batch"] * c["kv_heads"] * c["head_dim"]
        cache = rows * (c["held"] + c["new"] + c["prefix"])
        copied = rows * c["new"] if c["kind"] != "chunk" else 0
        pairs = c["batch"] * c["q_heads"] * c["new"] * (c["held"] + c["new"]) if c["kind"] == "chunk" else 0
        if cache * heavy <= MOST_CACHE and copied * heavy <= MOST_COPIED and pairs * heavy <= MOST_PAIRS:
            return c


def _esz(c):
    return 2 if c["dtype"] == "bf16" else 4


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _lens(c, seed):
    """Per sequence: tokens held, new tokens (-1, 0 where it sits out)."""
    B = c["batch"]
    if not c["ragged"]:
        return [c["held"]] * B, [c["new"]] * B
    r = random.Random(seed * 7919 + 1)
    held, new = [], []
    for b in range(B):
        out = b > 0 and r.random() < 0.25
        h, n = r.randint(c["held"] * 3 // 4, c["held"]), r.randint((c["new"] + 1) // 2, c["new"])
        held.append(-1 if out else max(h, n) if c["kind"] == "read" else h)
        new.append(0 if out else n)
    return held, new


def _starts(c, held, new):
    """First token that the call writes or reads."""
    return [max(0, h - n) if c["kind"] == "read" else max(0, h) for h, n in zip(held, new)]


def _width(c):
    """Pages of a sequence's row of the table."""
    return (c["held"] + (0 if c["kind"] == "read" else c["new"]) + c["page"] - 1) // c["page"]


def _inputs(c, seed):
    """Every input of the case, by name. Per sequence `held` tokens lie in front of the new ones."""
    device = _device()
    g = torch.Generator(device=device).manual_seed(seed)
    B, Hq, Hkv, d, dt = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], _dtype(c)
    L, n, S = c["held"], c["new"], c["prefix"]
    strong = torch.ones(Hkv, 1, d, device=device)
    strong.scatter_(2, torch.randint(0, d, (Hkv, 1, 4), generator=g, device=device), 6.0)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=device)

    x = {}
    if S:
        x["prefix_k"], x["prefix_v"] = (randn(Hkv, S, d) * strong).to(dt), randn(Hkv, S, d).to(dt)
    if L:
        x["held_k"] = torch.empty(B, Hkv, L, d, dtype=dt, device=device)
        x["held_v"] = torch.empty(B, Hkv, L, d, dtype=dt, device=device)
        for b in range(B):
            x["held_k"][b], x["held_v"][b] = randn(Hkv, L, d) * strong, randn(Hkv, L, d)
    if c["kind"] != "read":
        x["k"], x["v"] = (randn(B, Hkv, n, d) * strong).to(dt), randn(B, Hkv, n, d).to(dt)
    if c["kind"] in ("step", "chunk"):
        keys = x["held_k"] if L else x["k"]
        at = torch.randint(0, max(1, (L or n) * 3 // 4), (n,), generator=g, device=device)
        k = keys[:, :, at].float()  # [B, Hkv, n, d]
        q = randn(B, n, Hkv, Hq // Hkv, d) + 2.0 * (k / k.norm(dim=-1, keepdim=True)).transpose(1, 2).unsqueeze(3)
        x["q"] = q.reshape(B, n, Hq, d).to(dt)
    pages = B * _width(c)
    x["table"] = torch.randperm(pages, generator=g, device=device).reshape(B, _width(c)).to(torch.int32)
    return x


class _State:
    pass


def prepare(case, seed):
    c, x = case, _inputs(case, seed)
    s = _State()
    held, new = _lens(c, seed)
    s.case, s.x = c, x
    B, Hq, Hkv, d, n, kind = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["new"], c["kind"]
    L, pages = c["held"], c["batch"] * _width(c)

    def zeros(*shape, dtype=None):
        return torch.zeros(*shape, dtype=_dtype(c) if dtype is None else dtype, device=_device())

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=_device())

    s.held, s.new, s.start = ints(held), ints(new), ints(_starts(c, held, new))
    s.total = s.start + s.new
    at_start, before = ints([0] * B), ints([max(0, h) for h in held])
    if kind == "step":
        s.out = {"out": zeros(B, Hq, d), "lse": zeros(B, Hq, dtype=torch.float32), "k": zeros(B, Hkv, d),
                 "v": zeros(B, Hkv, d)}
    elif kind == "chunk":
        s.out = {"out": zeros(B, n, Hq, d), "lse": zeros(B, n, Hq, dtype=torch.float32)}
    else:
        s.out = {"k": zeros(B, Hkv, n, d), "v": zeros(B, Hkv, n, d)}
    if own:
        import paper_2502_11147_amd as raas

        s.prefix = None
        if c["prefix"]:
            s.prefix = raas.SharedPrefix(1, Hq, Hkv, d, max_tokens=c["prefix"], max_rows=B, dtype=c["dtype"])
            s.prefix.store(0, x["prefix_k"], x["prefix_v"])
        s.cache = raas.QuantCache(1, Hq, Hkv, d, n_pages=pages, page_size=c["page"], max_batch=B, max_queries=n,
                                  key_bits=c["key_bits"], value_bits=c["value_bits"], dtype=c["dtype"])
        if L:
            s.cache.write(0, x["held_k"], x["held_v"], x["table"], at_start, before)
        if kind == "step":
            s.args = s.cache.prepare_step(0, x["q"][:, 0].contiguous(), x["k"][:, :, 0].contiguous(),
                                          x["v"][:, :, 0].contiguous(), s.out["out"], x["table"], s.held,
                                          lse=s.out["lse"], k_held=s.out["k"], v_held=s.out["v"], prefix=s.prefix)
    else:
        bits = {"k": c["key_bits"], "v": c["value_bits"]}
        s.pool = {name: (torch.zeros(pages, Hkv, c["page"], d, dtype=torch.uint8, device=_device()),
                         torch.zeros(pages, Hkv, c["page"], d // 32, dtype=torch.uint8, device=_device())) for name in bits}
        s.value = {name: _values(bits[name]).to(device=_device(), dtype=torch.float32) for name in bits}
        for b in range(B if L else 0):
            _plain_write(s, x["held_k"][b:b + 1], x["held_v"][b:b + 1], at_start[b:b + 1], before[b:b + 1], b)
    if L:  # held in the cache from here on
        del x["held_k"], x["held_v"]
    return s


def run(state):
    s = state
    x, kind = s.x, s.case["kind"]
    if not own:
        if kind in ("store", "chunk"):
            _plain_write(s, x["k"], x["v"], s.start, s.new)
        if kind in ("store", "read"):
            return _plain_read(s)
        return _plain_step(s) if kind == "step" else _plain_attend(s)
    if kind == "step":
        s.cache.decode_prepared(s.args)
        return s.out
    if kind in ("store", "chunk"):
        s.cache.write(0, x["k"], x["v"], x["table"], s.start, s.new)
    if kind == "chunk":
        s.cache.attend(0, x["q"], s.out["out"], x["table"], s.total, counts=s.new, lse=s.out["lse"])
    else:
        s.cache.read(0, s.out["k"], s.out["v"], x["table"], s.start, s.new)
    return s.out


# ---------------------------------------------------------------------------
# The plain forms: elementary torch operations in 32 bits. Codes and the
# exponents of their groups lie in pages, a byte each.

def _values(bits):
    """The value of every code: sign, exponent, mantissa."""
    exp_bits, man_bits, bias = (2, 1, 1) if bits == 4 else (4, 3, 7)
    v = []
    for code in range(1 << bits):
        e, m = code >> man_bits & (1 << exp_bits) - 1, code & (1 << man_bits) - 1
        y = m * 2.0 ** (1 - bias - man_bits) if e == 0 else (1 + m / (1 << man_bits)) * 2.0 ** (e - bias)
        v.append(-y if code >> (bits - 1) else y)
    return torch.tensor(v, dtype=torch.float64)


def _plain_quantise(x, bits):
    """Codes [..., d] and biased exponents [..., d / 32] of x."""
    least, most_exp, most, half = (0, 2, 6.0, 0x200000) if bits == 4 else (-6, 8, 448.0, 0x180000)
    man_bits = 1 if bits == 4 else 3
    g = x.float().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    e = (g.abs().amax(-1).view(torch.int32) + half >> 23) - most_exp
    e = e.clamp(16, 252 if bits == 4 else 246)
    y = g * (254 - e << 23).view(torch.float32).unsqueeze(-1)  # exact: a power of two
    a = y.abs()
    binade = ((a.view(torch.int32) >> 23) - 127).clamp(min=least)  # the step there is 2^(binade - man_bits)
    step = (binade - man_bits + 127 << 23).view(torch.float32)
    a = (torch.round(a / step) * step).clamp(max=most)
    # the code of a value: its binade and mantissa, counted from the least one
    binade = ((a.view(torch.int32) >> 23) - 127).clamp(min=least)
    step = (binade - man_bits + 127 << 23).view(torch.float32)
    code = (a / step).int() + (binade - least << man_bits)
    code = code + (torch.signbit(g).int() << (bits - 1))
    return code.to(torch.uint8).reshape(x.shape), e.to(torch.uint8)


def _plain_write(s, k, v, start, count, seq0=0):
    """Tokens 0 .. count - 1 of each of k's sequences (seq0 on) become tokens start .. of the cache."""
    c = s.case
    t = torch.arange(k.shape[2], device=k.device)
    seq, tok = torch.nonzero(t < count[:, None], as_tuple=True)
    at = start.long()[seq] + tok
    page, row = s.x["table"].long()[seq + seq0, at // c["page"]], at % c["page"]
    for name, x in (("k", k), ("v", v)):
        code, e = _plain_quantise(x[seq, :, tok], c["key_bits"] if name == "k" else c["value_bits"])
        s.pool[name][0][page, :, row] = code
        s.pool[name][1][page, :, row] = e


def _plain_gather(s, name):
    """[B, Hkv, tokens of the table's pages, d] in 32 bits."""
    c, table = s.case, s.x["table"].long()
    code, e = (p[table].transpose(1, 2).flatten(2, 3) for p in s.pool[name])
    x = s.value[name][code.int()].unflatten(-1, (-1, 32))
    return (x * (e.int() << 23).view(torch.float32).unsqueeze(-1)).flatten(-2)


def _plain_read(s):
    c, n = s.case, s.case["new"]
    t = torch.arange(n, device=s.new.device)
    at = (s.start[:, None] + t).clamp(max=_width(c) * c["page"] - 1).long()
    rows = at[:, None, :, None].expand(c["batch"], c["kv_heads"], n, c["head_dim"])
    given = (t < s.new[:, None])[:, None, :, None]
    for name in ("k", "v"):
        s.out[name] = torch.where(given, _plain_gather(s, name).gather(2, rows).to(_dtype(c)), s.out[name])
    return s.out


def _plain_softmax(s, q, k, v, sees):
    """Numerators, maxima, sums of q [units, rows, d] over k, v [units, tokens, d]; sees: a mask or None."""
    x = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(q.shape[-1])
    if sees is not None:
        x.masked_fill_(~sees, -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-1e30)
    x = torch.exp(x.sub_(m))
    return torch.bmm(x, v), m, x.sum(-1, keepdim=True)


def _plain_step(s):
    c, x = s.case, s.x
    B, Hq, Hkv, d = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"]
    _plain_write(s, x["k"], x["v"], s.start, s.new)
    k, v = (_plain_gather(s, name) for name in ("k", "v"))
    tokens = k.shape[2]
    t = torch.arange(tokens, device=k.device)
    sees = (t <= s.held[:, None])[:, None, None].expand(B, Hkv, 1, tokens).reshape(B * Hkv, 1, tokens)
    q = x["q"].float().reshape(B, Hkv, Hq // Hkv, d)
    o, m, z = _plain_softmax(s, q.flatten(0, 1), k.flatten(0, 1), v.flatten(0, 1), sees)
    if c["prefix"]:
        qp = q.transpose(0, 1).reshape(Hkv, -1, d)
        parts = _plain_softmax(s, qp, x["prefix_k"].float(), x["prefix_v"].float(), None)
        op, mp, zp = (y.reshape(Hkv, B, Hq // Hkv, -1).transpose(0, 1).flatten(0, 1) for y in parts)
        most = torch.maximum(m, mp)
        o, z = o * torch.exp(m - most) + op * torch.exp(mp - most), z * torch.exp(m - most) + zp * torch.exp(mp - most)
        m = most
    on = (s.held >= 0)[:, None]
    last = s.held.clamp(min=0).long()[:, None, None, None].expand(B, Hkv, 1, d)
    r = {"out": (o / z.clamp(min=1e-30)).reshape(B, Hq, d).to(_dtype(c)),
         "lse": (m + torch.log(z.clamp(min=1e-30))).reshape(B, Hq),
         "k": k.gather(2, last)[:, :, 0].to(_dtype(c)), "v": v.gather(2, last)[:, :, 0].to(_dtype(c))}
    for name, y in r.items():
        s.out[name] = torch.where(on.reshape([B] + [1] * (y.dim() - 1)), y, s.out[name])
    return s.out


def _plain_attend(s):
    c, x = s.case, s.x
    B, Hq, Hkv, d, n = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["new"]
    k, v = (_plain_gather(s, name) for name in ("k", "v"))
    tokens = k.shape[2]
    t, i = torch.arange(tokens, device=k.device), torch.arange(n, device=k.device)
    given = i < s.new[:, None]
    for b in range(B):  # a sequence at a time: the logits of all would not fit
        sees = ((t <= s.start[b] + i[:, None]) & given[b][:, None])[None, :, None]
        sees = sees.expand(1, n, Hq // Hkv, tokens).reshape(1, -1, tokens)
        q = x["q"][b].float().reshape(n, Hkv, -1, d).transpose(0, 1).reshape(Hkv, -1, d)
        o, m, z = _plain_softmax(s, q, k[b], v[b], sees)
        o = (o / z.clamp(min=1e-30)).reshape(Hkv, n, -1, d).transpose(0, 1).reshape(n, Hq, d).to(_dtype(c))
        lse = (m + torch.log(z.clamp(min=1e-30))).reshape(Hkv, n, -1).transpose(0, 1).reshape(n, Hq)
        s.out["out"][b] = torch.where(given[b][:, None, None], o, s.out["out"][b])
        s.out["lse"][b] = torch.where(given[b][:, None], lse, s.out["lse"][b])
    return s.out


# ---------------------------------------------------------------------------
# The definition in 64 bits, sequence by sequence and head by head.

def _held_value(x, bits):
    """The value that the cache holds for x [..., d]: per group the least power of
    two X with max |x| < limit X, then the nearest of the type's values times X."""
    grid = torch.unique(_values(bits).abs()).to(x.device)  # in order; places with even numbers have even codes
    limit = 7.0 if bits == 4 else 464.0
    g = x.double().unflatten(-1, (-1, 32))
    most = g.abs().amax(-1, keepdim=True)
    e = torch.full_like(most, -111.0)
    for p in range(-40, 41):  # (the inputs lie well within)
        e = torch.where(most >= limit * 2.0 ** (p - 1), torch.full_like(e, float(p)), e)
    X = torch.exp2(e)
    y = g.abs() / X
    hi = torch.searchsorted(grid, y).clamp(max=len(grid) - 1)  # the first place at or above y
    lo = (hi - 1).clamp(min=0)
    below, above = y - grid[lo], grid[hi] - y
    place = torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return (torch.copysign(grid[place], g) * X).flatten(-2)


def exact(case, seed):
    c, x = case, _inputs(case, seed)
    held, new = _lens(c, seed)
    B, Hq, Hkv, d, n, kind = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["new"], c["kind"]
    G, scale = Hq // Hkv, 1.0 / math.sqrt(d)
    device = x["table"].device
    bits = {"k": c["key_bits"], "v": c["value_bits"]}

    def zeros(*shape):
        return torch.zeros(*shape, dtype=torch.float64, device=device)

    def tokens(name, b, h):
        """All tokens of one unit as they are held: those before, those of the call."""
        parts = [x["held_" + name][b, h, :held[b]]] if c["held"] else []
        if kind != "read":
            parts.append(x[name][b, h, :new[b]])
        return _held_value(torch.cat(parts), bits[name])

    if kind in ("store", "read"):
        r = {"k": zeros(B, Hkv, n, d), "v": zeros(B, Hkv, n, d)}
        for b in range(B):
            for h in range(Hkv):
                for name in r:
                    if new[b] > 0:
                        r[name][b, h, :new[b]] = tokens(name, b, h)[-new[b]:]
        return r
    out, lse = zeros(B, n, Hq, d), zeros(B, n, Hq)
    k_held, v_held = zeros(B, Hkv, d), zeros(B, Hkv, d)
    for b in range(B):
        if new[b] == 0:
            continue
        for h in range(Hkv):
            k, v = tokens("k", b, h), tokens("v", b, h)
            k_held[b, h], v_held[b, h] = k[-1], v[-1]
            total = len(k)
            if c["prefix"]:
                k, v = torch.cat([k, x["prefix_k"][h].double()]), torch.cat([v, x["prefix_v"][h].double()])
            heads = slice(h * G, (h + 1) * G)
            for i0 in range(0, new[b], 256):
                i1 = min(new[b], i0 + 256)
                q = x["q"][b, i0:i1, heads].double()
                a = torch.matmul(q.reshape(-1, d), k.t().contiguous()).reshape(i1 - i0, G, -1) * scale
                if kind == "chunk":
                    last = total - new[b] + torch.arange(i0, i1, device=device)
                    a = a.masked_fill((torch.arange(total, device=device) > last[:, None])[:, None], -math.inf)
                lse[b, i0:i1, heads] = torch.logsumexp(a, 2)
                out[b, i0:i1, heads] = torch.matmul(torch.softmax(a, 2), v)
    if kind == "step":
        return {"out": out[:, 0], "lse": lse[:, 0], "k": k_held, "v": v_held}
    return {"out": out, "lse": lse}


def work(case):
    """One pass: what is written and read of the cache once, new keys and values,
    queries and outputs once, and one pair of products per query head and token
    that it sees."""
    c = case
    e, d, Hq, Hkv = _esz(c), c["head_dim"], c["q_heads"], c["kv_heads"]
    token = Hkv * (d * (c["key_bits"] + c["value_bits"]) / 8.0 + d / 16.0)
    rows = 2.0 * Hkv * d * e
    b = f = 0.0
    for held, new in zip(*_lens(c, 0)):
        if c["kind"] in ("store", "read"):
            b += new * (rows + token) * (2 if c["kind"] == "store" else 1)
        elif new > 0:
            b += (held + 2 * new) * token + new * (rows + 2 * Hq * d * e + 4 * Hq)
            b += rows if c["kind"] == "step" else 0
            f += 4.0 * Hq * d * (new * (held + c["prefix"]) + new * (new + 1) / 2.0)
    return {"bytes": b + 2.0 * Hkv * c["prefix"] * d * e, "flops": f}
