"""The cache that evicts by accumulated attention weight, the shared prefix and
the prompt weights (second half of ``include/raas.h``) -- argument marshalling
only. Tensors lie on the device that was current when the handle was made (for
prompt_weights, on q's), streams default to that device's current one."""
from __future__ import annotations

import ctypes

from . import BF16, F32, _check, _torch, load_library


class WeightConfig(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in
                ("batch", "n_layers", "n_q_heads", "n_kv_heads", "head_dim", "capacity", "recent", "dtype")]


class PrefixConfig(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in
                ("n_layers", "n_q_heads", "n_kv_heads", "head_dim", "max_tokens", "max_rows", "dtype")]


def _dtype_code(dtype: str) -> int:
    if dtype not in ("bf16", "f32"):
        raise ValueError("dtype must be 'bf16' or 'f32' (got %r)" % (dtype,))
    return BF16 if dtype == "bf16" else F32


def _pointer(t, name, dtype, shape, device, optional=False):
    """Address of a contiguous device tensor of this type, shape and device index."""
    if t is None and optional:
        return None
    try:
        if t.get_device() == device and t.dtype is dtype and t.shape == shape and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    if not isinstance(t, _torch().Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) tensor" % name)
    raise ValueError("%s must be a contiguous %s tensor of shape %s on cuda:%d (got %s %s on %s)"
                     % (name, dtype, tuple(shape), device, t.dtype, tuple(t.shape), t.device))


def _stream(stream, device):
    if stream is None:
        stream = _torch().cuda.current_stream(device)
    return stream.cuda_stream


def _host_ints(values, n, name):
    """A C int32 array of n host values, or None."""
    if values is None:
        return None
    values = [int(x) for x in values]
    if len(values) != n:
        raise ValueError("%s must have %d entries" % (name, n))
    return (ctypes.c_int32 * n)(*values)


class _Handle:
    """A C handle, the type and the device of its tensors."""

    _destroy = None

    def __init__(self, create, config, dtype: str, stream):
        torch = _torch()
        self.lib = load_library()
        self.cfg, self.dtype = config, dtype
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self._float32, self._int32 = torch.float32, torch.int32
        self.device = torch.cuda.current_device()
        self._h = ctypes.c_void_p()
        _check(getattr(self.lib, create)(ctypes.byref(config), _stream(stream, self.device), ctypes.byref(self._h)),
               create)

    def close(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value:
            getattr(self.lib, self._destroy)(h)
            h.value = None  # prepared steps hold this object

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def handle(self):
        return self._h

    def _tensor(self, t, shape, name, optional=False):
        return _pointer(t, name, self.torch_dtype, shape, self.device, optional)

    def _floats(self, t, shape, name):
        return _pointer(t, name, self._float32, shape, self.device, optional=True)

    def _ints(self, t, shape, name):
        return _pointer(t, name, self._int32, shape, self.device, optional=True)


class SharedPrefix(_Handle):
    """A prompt that a batch shares, stored once per layer (raas_create_prefix)."""

    _destroy = "raas_destroy_prefix"

    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, max_tokens: int, max_rows: int,
                 dtype: str = "bf16", stream=None):
        self.n_layers, self.n_q_heads, self.n_kv_heads, self.head_dim = n_layers, n_q_heads, n_kv_heads, head_dim
        super().__init__("raas_create_prefix", PrefixConfig(n_layers, n_q_heads, n_kv_heads, head_dim, max_tokens,
                                                            max_rows, _dtype_code(dtype)), dtype, stream)

    def store(self, layer: int, k, v, stream=None):
        """k, v: [n_kv_heads][tokens][head_dim] device tensors, or None for an
        empty prefix (raas_prefix_store)."""
        tokens = 0 if k is None else int(k.shape[1])
        shape = (self.n_kv_heads, tokens, self.head_dim)
        kp = self._tensor(k, shape, "k") if tokens else None
        vp = self._tensor(v, shape, "v") if tokens else None
        _check(self.lib.raas_prefix_store(self._h, layer, kp, vp, tokens, _stream(stream, self.device)),
               "raas_prefix_store")

    def attend(self, layer: int, q, out, lse=None, stream=None):
        """Attention of q [rows][n_q_heads][head_dim] over the layer's prefix
        into out (same shape) and lse (fp32 [rows][n_q_heads], optional)
        (raas_prefix_attention)."""
        rows = q.shape[0]
        shape = (rows, self.n_q_heads, self.head_dim)
        qp, op = self._tensor(q, shape, "q"), self._tensor(out, shape, "out")
        lp = self._floats(lse, shape[:2], "lse")
        _check(self.lib.raas_prefix_attention(self._h, layer, qp, rows, op, lp, _stream(stream, self.device)),
               "raas_prefix_attention")

    def device_bytes(self) -> int:
        return int(self.lib.raas_prefix_bytes(self._h))


class PreparedStep(tuple):
    """The arguments of one raas_weight_step call; keeps its tensors and its prefix."""

    prefix = None
    tensors = ()


class WeightCache(_Handle):
    """A cache that evicts the token of least accumulated attention weight
    (raas_create_weight_cache)."""

    _destroy = "raas_destroy_weight_cache"

    def __init__(self, batch: int, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, capacity: int,
                 recent: int, dtype: str = "bf16", stream=None):
        self.batch, self.n_layers, self.capacity, self.recent = batch, n_layers, capacity, recent
        self.n_q_heads, self.n_kv_heads, self.head_dim = n_q_heads, n_kv_heads, head_dim
        self.units = batch * n_kv_heads
        super().__init__("raas_create_weight_cache", WeightConfig(batch, n_layers, n_q_heads, n_kv_heads, head_dim,
                                                                  capacity, recent, _dtype_code(dtype)), dtype, stream)

    def prefill(self, layer: int, k, v, lens=None, weights=None, mask=None, stream=None):
        """(Re)starts sequences with their prompts (raas_weight_prefill). k, v:
        [batch][n_kv_heads][max_len][head_dim] device tensors, or None for empty
        prompts; weights: fp32 [batch][n_kv_heads][max_len] or None; lens, mask:
        host sequences of batch ints (None: full length; every sequence)."""
        B = self.batch
        max_len = 0 if k is None else int(k.shape[2])
        shape = (B, self.n_kv_heads, max_len, self.head_dim)
        kp = self._tensor(k, shape, "k") if max_len else None
        vp = self._tensor(v, shape, "v") if max_len else None
        wp = self._floats(weights, shape[:3], "weights") if max_len else None
        _check(self.lib.raas_weight_prefill(self._h, layer, kp, vp, wp, _host_ints(lens, B, "lens"),
                                            _host_ints(None if mask is None else [bool(x) for x in mask], B, "mask"),
                                            max_len, _stream(stream, self.device)), "raas_weight_prefill")

    def prepare_step(self, layer: int, q, k_new, v_new, out, positions=None, weights=None, evicted=None, stream=None,
                     active=None, prefix=None) -> PreparedStep:
        """Checks and converts the arguments of one raas_weight_step call once,
        so a loop can replay them with decode_prepared(). positions, evicted:
        int32 [batch][n_kv_heads][capacity] and [batch][n_kv_heads]; weights:
        fp32 like positions; active: int32 [batch]; all optional device tensors.
        prefix: a SharedPrefix, or None."""
        B, Hq, Hkv, d, C = self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, self.capacity
        if prefix is not None and not isinstance(prefix, SharedPrefix):
            raise TypeError("prefix must be a SharedPrefix")
        step = PreparedStep((
            self._h, layer,
            self._tensor(q, (B, Hq, d), "q"),
            self._tensor(k_new, (B, Hkv, d), "k_new"),
            self._tensor(v_new, (B, Hkv, d), "v_new"),
            self._tensor(out, (B, Hq, d), "out"),
            self._ints(positions, (B, Hkv, C), "positions"),
            self._floats(weights, (B, Hkv, C), "weights"),
            self._ints(evicted, (B, Hkv), "evicted"),
            self._ints(active, (B,), "active"),
            None if prefix is None else prefix.handle,
            _stream(stream, self.device),
        ))
        step.prefix = prefix
        step.tensors = (q, k_new, v_new, out, positions, weights, evicted, active)
        return step

    def decode_prepared(self, step: PreparedStep):
        if step.prefix is not None and not step.prefix.handle.value:
            raise ValueError("the step's prefix is closed")
        _check(self.lib.raas_weight_step(*step), "raas_weight_step")

    def decode_step(self, layer: int, q, k_new, v_new, out, positions=None, weights=None, evicted=None, stream=None,
                    active=None, prefix=None):
        """One decode step of one layer (raas_weight_step)."""
        self.decode_prepared(self.prepare_step(layer, q, k_new, v_new, out, positions, weights, evicted, stream, active,
                                               prefix))

    def export_state(self, layer: int, stream=None) -> dict:
        """Positions and weights [units][capacity] and clocks [units] as host
        arrays (raas_weight_export_state)."""
        import numpy as np

        pos = np.empty((self.units, self.capacity), np.int32)
        w = np.empty((self.units, self.capacity), np.float32)
        clock = np.empty(self.units, np.int32)
        ip = ctypes.POINTER(ctypes.c_int32)
        _check(self.lib.raas_weight_export_state(self._h, layer, pos.ctypes.data_as(ip),
                                                 w.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                                                 clock.ctypes.data_as(ip), _stream(stream, self.device)),
               "raas_weight_export_state")
        return dict(positions=pos, weights=w, clock=clock)

    def device_bytes(self) -> int:
        return int(self.lib.raas_weight_cache_bytes(self._h))


def prompt_weights(q, k, weights, lens=None, prefix_lse=None, stream=None):
    """The attention weights that a prompt's last queries give its tokens
    (raas_prompt_weights). q: [batch][window][n_q_heads][head_dim]; k:
    [batch][n_kv_heads][max_len][head_dim] of the same type (bf16 or fp32);
    weights: fp32 [batch][n_kv_heads][max_len], written up to each length; lens:
    host sequence of batch ints, or None; prefix_lse: fp32
    [batch][window][n_q_heads], or None."""
    torch = _torch()
    lib = load_library()
    if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dim() != 4:
        raise TypeError("q must be a CUDA (HIP) tensor [batch][window][n_q_heads][head_dim]")
    if q.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("q must be bfloat16 or float32 (got %s)" % q.dtype)
    if not isinstance(k, torch.Tensor) or k.dim() != 4:
        raise TypeError("k must be a CUDA (HIP) tensor [batch][n_kv_heads][max_len][head_dim]")
    (B, W, Hq, d), (Hkv, P), dev = q.shape, k.shape[1:3], q.device.index
    code = BF16 if q.dtype == torch.bfloat16 else F32
    qp, kp = _pointer(q, "q", q.dtype, (B, W, Hq, d), dev), _pointer(k, "k", q.dtype, (B, Hkv, P, d), dev)
    wp = _pointer(weights, "weights", torch.float32, (B, Hkv, P), dev)
    lp = _pointer(prefix_lse, "prefix_lse", torch.float32, (B, W, Hq), dev, optional=True)
    need = int(lib.raas_prompt_weights_workspace(B, Hq, Hkv, P, W))
    current = torch.cuda.current_stream(dev)
    if stream is None:
        stream = current

    def call():
        space = torch.empty(max(need, 1), dtype=torch.uint8, device=q.device)
        _check(lib.raas_prompt_weights(B, Hq, Hkv, d, code, qp, kp, lp, _host_ints(lens, B, "lens"), P, W, wp,
                                       space.data_ptr(), need, stream.cuda_stream),
               "raas_prompt_weights")

    if dev == torch.cuda.current_device() and stream == current:
        call()
    else:  # (the workspace belongs to the stream that uses it)
        with torch.cuda.device(dev), torch.cuda.stream(stream):
            call()
