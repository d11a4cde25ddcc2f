"""The weight cache's fp64 statement against the repository's own heavy-hitter
oracle, and the refusals of the C entry points (no GPU)."""
from __future__ import annotations

import ctypes
import os
import re

import numpy as np
import pytest

import weight_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("recent", [0, 3, 11])
@pytest.mark.parametrize("P", [0, 5, 12, 30])
def test_statement_is_the_heavy_hitter_policy(P, recent):
    """The cache evicts when the next token arrives, the oracle when it has
    stored one: the same tokens are attended."""
    from oracle import baselines

    rng = np.random.default_rng(P)
    G, d, L = 3, 16, 12
    K, V = rng.standard_normal((P, d)), rng.standard_normal((P, d))
    u = ref.Unit(G, d, L, recent, False)
    u.start(K, V, None)
    h = baselines.H2O(K, V, L, recent)
    for _ in range(40):
        q, k, v = rng.standard_normal((G, d)), rng.standard_normal(d), rng.standard_normal(d)
        out, att = h.step(q, k, v)
        assert np.abs(u.step(q, k, v)[0] - out).max() < 1e-12
        assert sorted(att) == sorted(u.pos[u.pos >= 0])


def test_prompt_weights_statement():
    """Column sums of the causal softmax, from the whole matrix."""
    rng = np.random.default_rng(1)
    n, G, d = 23, 2, 8
    q, k = rng.standard_normal((n, G, d)), rng.standard_normal((n, d))
    x = np.einsum("igd,jd->gij", q, k) / np.sqrt(d)
    x[:, np.arange(n)[:, None] < np.arange(n)] = -np.inf
    a = np.exp(x - x.max(-1, keepdims=True))
    a /= a.sum(-1, keepdims=True)
    assert np.abs(ref.prompt_weights(q, k)[0] - a.sum((0, 1))).max() < 1e-12
    assert np.abs(ref.prompt_weights(q[-5:], k)[0] - a[:, -5:].sum((0, 1))).max() < 1e-12
    lse = rng.standard_normal((n, G))
    z = np.exp(lse.T) / (np.exp(lse.T) + np.exp(np.where(np.isinf(x), -np.inf, x)).sum(-1))
    want = (a * (1.0 - z)[..., None]).sum((0, 1))
    assert np.abs(ref.prompt_weights(q, k, lse)[0] - want).max() < 1e-12


@pytest.fixture(scope="module")
def lib():
    import paper_2502_11147_amd as raas

    if not os.path.exists(raas.LIB_PATH):
        from paper_2502_11147_amd import build as b

        b.build()
    return raas.load_library()


@pytest.mark.parametrize("name,struct", [("raas_weight_config", "WeightConfig"), ("raas_prefix_config", "PrefixConfig")])
def test_config_layouts_match_the_header(name, struct):
    import paper_2502_11147_amd as raas

    text = open(os.path.join(ROOT, "include", "raas.h")).read()
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, text).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields = [f.strip() for decl in re.findall(r"int32_t ([^;]+);", body) for f in decl.split(",")]
    assert [(f, ctypes.c_int32) for f in fields] == getattr(raas, struct)._fields_


HEADS = [dict(n_kv_heads=0), dict(n_kv_heads=65536, n_q_heads=65536), dict(n_q_heads=7), dict(n_q_heads=0),
         dict(n_q_heads=34), dict(head_dim=96), dict(head_dim=0), dict(dtype=2), dict(dtype=-1), dict(n_layers=0)]
CACHE = HEADS + [dict(batch=0), dict(capacity=1), dict(capacity=(1 << 20) + 1), dict(recent=-1), dict(recent=64),
                 dict(batch=1 << 20)]
PREFIX = HEADS + [dict(max_tokens=0), dict(max_tokens=(1 << 20) + 1), dict(max_rows=0), dict(max_rows=1 << 22)]
PROMPT = HEADS[:-1] + [dict(batch=0), dict(max_len=-1), dict(max_len=(1 << 20) + 1), dict(window=0), dict(window=65),
                       dict(lens=(64, 65)), dict(lens=(-1, 3)), dict(q=None), dict(k=None), dict(weights=None),
                       dict(workspace=None), dict(space=1),
                       dict(n_q_heads=32, max_len=1 << 20, window=1 << 20)]
_ids = lambda bad: ",".join("%s=%s" % kv for kv in bad.items())  # noqa: E731


@pytest.mark.parametrize("bad", CACHE, ids=_ids)
def test_cache_refuses(lib, bad):
    import paper_2502_11147_amd as raas

    cfg = dict(batch=2, n_layers=1, n_q_heads=8, n_kv_heads=2, head_dim=128, capacity=64, recent=16, dtype=raas.BF16)
    cfg.update(bad)
    h = ctypes.c_void_p()
    assert lib.raas_create_weight_cache(ctypes.byref(raas.WeightConfig(**cfg)), None, ctypes.byref(h)) == raas.E_INVALID
    assert not h.value and raas.last_error()


@pytest.mark.parametrize("bad", PREFIX, ids=_ids)
def test_prefix_refuses(lib, bad):
    import paper_2502_11147_amd as raas

    cfg = dict(n_layers=1, n_q_heads=8, n_kv_heads=2, head_dim=128, max_tokens=64, max_rows=4, dtype=raas.BF16)
    cfg.update(bad)
    h = ctypes.c_void_p()
    assert lib.raas_create_prefix(ctypes.byref(raas.PrefixConfig(**cfg)), None, ctypes.byref(h)) == raas.E_INVALID
    assert not h.value and raas.last_error()


@pytest.mark.parametrize("bad", PROMPT, ids=_ids)
def test_prompt_weights_refuses(lib, bad):
    """(the pointers are never followed: each call is refused before a launch)"""
    import paper_2502_11147_amd as raas

    a = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=raas.BF16, q=64, k=64, lens=(64, 3), max_len=64,
             window=64, weights=64, workspace=64, space=1 << 30)
    a.update(bad)
    lens = (ctypes.c_int32 * 2)(*a["lens"])
    rc = lib.raas_prompt_weights(a["batch"], a["n_q_heads"], a["n_kv_heads"], a["head_dim"], a["dtype"], a["q"], a["k"],
                                 None, lens, a["max_len"], a["window"], a["weights"], a["workspace"], a["space"], None)
    assert rc == raas.E_INVALID and raas.last_error()


def test_null_handles(lib):
    import paper_2502_11147_amd as raas

    h = ctypes.c_void_p()
    assert lib.raas_create_weight_cache(None, None, ctypes.byref(h)) == raas.E_INVALID
    assert lib.raas_create_weight_cache(None, None, None) == raas.E_INVALID
    assert lib.raas_create_prefix(None, None, ctypes.byref(h)) == raas.E_INVALID
    assert lib.raas_create_prefix(None, None, None) == raas.E_INVALID
    assert lib.raas_weight_prefill(None, 0, None, None, None, None, None, 0, None) == raas.E_INVALID
    assert lib.raas_weight_step(None, 0, *[None] * 10) == raas.E_INVALID
    assert lib.raas_weight_export_state(None, 0, None, None, None, None) == raas.E_INVALID
    assert lib.raas_prefix_store(None, 0, None, None, 0, None) == raas.E_INVALID
    assert lib.raas_prefix_attention(None, 0, None, 0, None, None, None) == raas.E_INVALID
    assert lib.raas_weight_cache_bytes(None) == lib.raas_prefix_bytes(None) == 0
    assert lib.raas_prompt_weights_workspace(0, 8, 2, 64, 64) == 0
    assert lib.raas_prompt_weights_workspace(1, 7, 2, 64, 64) == 0
    lib.raas_destroy_weight_cache(None)
    lib.raas_destroy_prefix(None)
