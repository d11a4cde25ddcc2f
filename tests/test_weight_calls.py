"""Calls around the weight cache that other tests leave out: sizes that a query
must refuse, handles past 64 bits, workspaces of any float alignment, the count
of what is read, the README's example."""
from __future__ import annotations

import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2502_11147_amd as raas

    if not os.path.exists(raas.LIB_PATH):
        from paper_2502_11147_amd import build as b

        b.build()
    return raas.load_library()


# batch, query heads, KV heads, max_len, window
REFUSED = [(0, 8, 2, 64, 64), (1, 7, 2, 64, 64), (1, 0, 1, 64, 64), (1, 1, 0, 64, 64), (1, 34, 2, 64, 64),
           (1, 65536, 65536, 64, 64), (1, 8, 2, -1, 1), (1, 8, 2, (1 << 20) + 1, 64), (1, 8, 2, 2 ** 31 - 1, 64),
           (1, 8, 2, 64, 0), (1, 8, 2, 64, 65), (1, 8, 2, 64, 2 ** 31 - 1), (1, 16, 1, 1 << 20, 1 << 20)]


@pytest.mark.parametrize("sizes", REFUSED)
def test_workspace_of_refused_sizes_is_zero(lib, sizes):
    """The query and the call refuse the same sizes (the pointers are not followed)."""
    import paper_2502_11147_amd as raas

    assert lib.raas_prompt_weights_workspace(*sizes) == 0
    batch, hq, hkv, max_len, window = sizes
    assert lib.raas_prompt_weights(batch, hq, hkv, 64, raas.F32, 64, 64, None, None, max_len, window, 64, 64, 1 << 40,
                                   None) == raas.E_INVALID


@pytest.mark.parametrize("sizes", [(1, 1, 1, 1, 1), (3, 14, 2, 700, 9), (1, 16, 1, 1 << 20, 1 << 19), (1, 65535, 65535, 8, 8)])
def test_workspace_of_allowed_sizes(lib, sizes):
    assert lib.raas_prompt_weights_workspace(*sizes) > 0
    assert lib.raas_prompt_weights_workspace(*sizes[:3], 0, 1) == 0  # nothing to do


# sizes of which the product, or that of the keys alone, is 0 or small modulo 2^64
@pytest.mark.parametrize("layers,kv_heads", [(1 << 20, 32768), ((1 << 20) + 1, 32768), (1 << 21, 32768), (1 << 19, 65535)])
def test_prefix_of_more_bytes_than_64_bits_count(lib, layers, kv_heads):
    import paper_2502_11147_amd as raas

    cfg = raas.PrefixConfig(layers, kv_heads, kv_heads, 128, 1 << 20, 1, raas.F32)
    h = ctypes.c_void_p()
    assert lib.raas_create_prefix(ctypes.byref(cfg), None, ctypes.byref(h)) == raas.E_OOM
    assert not h.value and b"bytes" in lib.raas_last_error()


@pytest.mark.parametrize("layers,batch", [(1 << 16, 1 << 19), (1 << 20, 1 << 15)])
def test_cache_of_more_bytes_than_64_bits_count(lib, layers, batch):
    import paper_2502_11147_amd as raas

    cfg = raas.WeightConfig(batch, layers, 1, 1, 128, 1 << 20, 0, raas.F32)
    h = ctypes.c_void_p()
    assert lib.raas_create_weight_cache(ctypes.byref(cfg), None, ctypes.byref(h)) == raas.E_OOM
    assert not h.value and b"bytes" in lib.raas_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("shift", [1, 2, 3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_workspace_of_any_float_alignment(dtype, shift):
    """Seven heads and a window of one: the pairs of a row's maximum and sum
    start at an odd float; so do they behind a shifted workspace. The same bits."""
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_11147_amd as raas

    lib = raas.load_library()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(shift)
    P = 2100  # several pieces of the keys
    q, k = (torch.randn(*s, generator=g, device="cuda").to(dt) for s in ((1, 1, 7, 64), (1, 7, P, 64)))
    want, got = torch.zeros(1, 7, P, device="cuda"), torch.zeros(1, 7, P, device="cuda")
    raas.prompt_weights(q, k, want)
    need = lib.raas_prompt_weights_workspace(1, 7, 7, P, 1)
    space = torch.full((need // 4 + shift,), float("nan"), device="cuda")
    rc = lib.raas_prompt_weights(1, 7, 7, 64, raas.BF16 if dtype == "bf16" else raas.F32, q.data_ptr(), k.data_ptr(), None,
                                 None, P, 1, got.data_ptr(), space[shift:].data_ptr(), need,
                                 torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == 0 and torch.equal(want, got) and abs(float(got.sum()) - 7.0) < 1e-3


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tokens", [("bf16", 1000), ("f32", 70)])
def test_reads_of_a_prefix_are_counted(dtype, tokens):
    """What attention over a prefix reads is counted beside the steps' reads, by
    which a step tells whether its layer is still in the memory-side cache; a
    captured call is not."""
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_11147_amd as raas

    count = raas.load_library()._ZN4raas14count_streamedEiy
    count.restype, count.argtypes = ctypes.c_ulonglong, [ctypes.c_int, ctypes.c_ulonglong]
    B, Hq, Hkv, d, C = 3, 4, 2, 64, 40
    dt, block = (torch.bfloat16, 32) if dtype == "bf16" else (torch.float32, 16)
    size = 2 if dtype == "bf16" else 4
    p = raas.SharedPrefix(2, Hq, Hkv, d, tokens, B, dtype)
    c = raas.WeightCache(B, 2, Hq, Hkv, d, C, 4, dtype)
    kv = torch.randn(Hkv, tokens, d, device="cuda").to(dt)
    q, k = torch.randn(B, Hq, d, device="cuda").to(dt), torch.randn(B, Hkv, d, device="cuda").to(dt)
    out = torch.empty_like(q)
    p.store(1, kv, kv)
    c.prefill(1, None, None)
    reads = 2 * Hkv * -(-tokens // block) * block * d * size
    own = 2 * B * Hkv * -(-C // block) * block * d * size

    def counted(call):
        before = count(0, 0)
        call()
        return count(0, 0) - before

    assert counted(lambda: p.attend(1, q, out)) == reads
    assert counted(lambda: c.decode_step(1, q, k, k, out)) == own
    assert counted(lambda: c.decode_step(1, q, k, k, out, prefix=p)) == own + reads
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()

    def capture():
        with torch.cuda.graph(graph):
            p.attend(1, q, out)
            c.decode_step(1, q, k, k, out, prefix=p)

    assert counted(capture) == 0
    graph.replay()
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_readme_example():
    """The README's run of the three together, as it stands there: a private
    prompt's weights count the shared prompt in front of it, as the steps do."""
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import numpy as np

    import paper_2502_11147_amd as raas
    import weight_reference as ref

    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        blocks = f.read().split("```python\n")[1:]
    (code,) = [b.split("```")[0] for b in blocks if "SharedPrefix" in b]
    g = torch.Generator(device="cuda").manual_seed(1)
    mk = lambda *shape: torch.randn(*shape, generator=g, device="cuda").bfloat16()  # noqa: E731
    P, S, lens = 90, 200, [90 - i % 20 for i in range(64)]
    x = dict(raas=raas, k_shared=mk(8, S, 128), v_shared=mk(8, S, 128), q_prompt=mk(64, 64, 32, 128), k_prompt=mk(64, 8, P, 128),
             v_prompt=mk(64, 8, P, 128), o_prompt=mk(64 * 64, 32, 128), lse=torch.zeros(64 * 64, 32, device="cuda"),
             w=torch.zeros(64, 8, P, device="cuda"), lens=lens, q=mk(64, 32, 128), k_new=mk(64, 8, 128),
             v_new=mk(64, 8, 128), out=torch.full((64, 32, 128), float("nan"), device="cuda").bfloat16())
    exec(code, x)
    torch.cuda.synchronize()
    assert torch.isfinite(x["out"].float()).all()
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    for b, h in ((0, 0), (63, 7), (19, 3)):
        n, heads = lens[b], slice(4 * h, 4 * h + 4)
        Q = f64(x["q_prompt"][b, :, heads])
        lse = ref.prefix_attention(Q.reshape(-1, 128), f64(x["k_shared"][h]), f64(x["v_shared"][h]), True)
        want, bound = ref.prompt_weights(Q, f64(x["k_prompt"][b, h, :n]), lse[2].reshape(64, 4))
        # (the log-sum-exp that the call was given is off by its own bound, and a probability by as much)
        assert (np.abs(f64(x["w"][b, h, :n]) - want) <= bound + 2 * lse[3].max() * want).all()


def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_11147_amd as raas

    return torch, raas


@pytest.mark.gpu
def test_no_handle_is_created_during_capture():
    torch, raas = _gpu()
    x = torch.zeros(4, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        x += 1.0
        for make in (lambda: raas.WeightCache(1, 1, 4, 1, 64, 40, 4), lambda: raas.SharedPrefix(1, 4, 1, 64, 40, 4)):
            with pytest.raises(raas.RaasError) as e:
                make()
            assert e.value.code == raas.E_STATE
    graph.replay()  # the capture went on
    torch.cuda.synchronize()
    assert (x == 1.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [2, 20, 70])
def test_prefix_replays_over_other_lengths(rows):
    """A captured call keeps the number of parts of its capture, whatever is
    stored when it is replayed: longer, shorter, nothing, with and between eager
    calls."""
    torch, raas = _gpu()
    Hq, Hkv, d = 4, 2, 128
    g = torch.Generator(device="cuda").manual_seed(rows)
    mk = lambda *shape: torch.randn(*shape, generator=g, device="cuda").bfloat16()  # noqa: E731
    p = raas.SharedPrefix(1, Hq, Hkv, d, 3000, rows)
    q, out, want = mk(rows, Hq, d), mk(rows, Hq, d), mk(rows, Hq, d)
    lse, lse_want = torch.zeros(rows, Hq, device="cuda"), torch.zeros(rows, Hq, device="cuda")
    p.store(0, mk(Hkv, 1500, d), mk(Hkv, 1500, d))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        p.attend(0, q, out, lse)
    for n in (1500, 3000, 17, 0, 1, 33, 0, 2999):
        k, v = (mk(Hkv, n, d), mk(Hkv, n, d)) if n else (None, None)
        p.store(0, k, v)
        out.fill_(5.0)
        for _ in range(2):
            graph.replay()
        p.attend(0, q, want, lse_want)
        torch.cuda.synchronize()
        if n == 0:
            assert (out == 0).all() and (lse == -float("inf")).all()
        # (one bf16 rounding of either; the parts are added in another order)
        assert ((out.float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 1e-5).all(), n
        assert n == 0 or ((lse - lse_want).abs() <= 1e-5 * (1.0 + lse_want.abs())).all(), n
