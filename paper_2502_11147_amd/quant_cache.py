"""The quantised cache (last part of ``include/raas.h``) -- argument marshalling
only. Tensors lie on the device that was current when the handle was made, streams
default to that device's current one."""
from __future__ import annotations

import ctypes

from . import _check, _torch, load_library
from .weight_cache import SharedPrefix, _dtype_code, _Handle, _stream


class QuantConfig(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in
                ("n_layers", "n_q_heads", "n_kv_heads", "head_dim", "page_size", "n_pages", "max_batch", "max_queries",
                 "key_bits", "value_bits", "dtype")]


class PreparedQuantStep(tuple):
    """The arguments of one raas_quant_step call; keeps its tensors and its prefix."""

    prefix = None
    tensors = ()


class QuantCache(_Handle):
    """A paged cache of every token in 4 or 8 bits (raas_create_quant_cache)."""

    _destroy = "raas_destroy_quant_cache"

    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, n_pages: int, page_size: int = 64,
                 max_batch: int = 1, max_queries: int = 1, key_bits: int = 4, value_bits: int = 4, dtype: str = "bf16",
                 stream=None):
        self.n_layers, self.n_q_heads, self.n_kv_heads, self.head_dim = n_layers, n_q_heads, n_kv_heads, head_dim
        self.n_pages, self.page_size, self.max_batch, self.max_queries = n_pages, page_size, max_batch, max_queries
        self.key_bits, self.value_bits = key_bits, value_bits
        self._write, self._read = (getattr(load_library(), "raas_quant_" + x) for x in ("write", "read"))
        self._current_stream = _torch().cuda.current_stream
        super().__init__("raas_create_quant_cache",
                         QuantConfig(n_layers, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_batch,
                                     max_queries, key_bits, value_bits, _dtype_code(dtype)), dtype, stream)

    def _table(self, table, batch):
        """Address and width of the table of a call's sequences."""
        shape = getattr(table, "shape", ())
        width = shape[1] if len(shape) == 2 else 0
        address = self._ints(table, (batch, width), "table")
        if address is None:
            raise TypeError("table must be a CUDA (HIP) tensor")
        return address, width

    def _lengths(self, t, batch, name):
        address = self._ints(t, (batch,), name)
        if address is None:
            raise TypeError("%s must be a CUDA (HIP) tensor" % name)
        return address

    def _copy(self, call, name, layer, k, v, table, start, counts, stream):
        shape = getattr(k, "shape", ())
        if len(shape) != 4:
            raise TypeError("k must be a CUDA (HIP) tensor [batch][n_kv_heads][tokens][head_dim]")
        B, tokens = shape[0], shape[2]
        shape = (B, self.n_kv_heads, tokens, self.head_dim)
        kp, vp = self._tensor(k, shape, "k"), self._tensor(v, shape, "v")
        tp, width = self._table(table, B)
        if stream is None:
            stream = self._current_stream(self.device)
        rc = call(self._h, layer, kp, vp, tp, width, self._lengths(start, B, "start"), self._ints(counts, (B,), "counts"), B,
                  tokens, stream.cuda_stream)
        _check(rc, name)

    def write(self, layer: int, k, v, table, start, counts=None, stream=None):
        """Quantises and stores new tokens (raas_quant_write). k, v:
        [batch][n_kv_heads][tokens][head_dim]; table: int32 [batch][width], the pages
        of each sequence; start: int32 [batch], position of each sequence's first new
        token; counts: int32 [batch], how many of the rows (None: all). All device
        tensors."""
        self._copy(self._write, "raas_quant_write", layer, k, v, table, start, counts, stream)

    def read(self, layer: int, k, v, table, start, counts=None, stream=None):
        """Reads held tokens back into k, v (raas_quant_read); arguments as write."""
        self._copy(self._read, "raas_quant_read", layer, k, v, table, start, counts, stream)

    def attend(self, layer: int, q, out, table, lens, counts=None, lse=None, stream=None):
        """Causal attention of the last tokens' queries over what their sequences hold
        (raas_quant_attention). q, out: [batch][queries][n_q_heads][head_dim]; lens:
        int32 [batch], tokens held, those of the queries among them; counts: int32
        [batch], how many of the rows (None: all); lse: fp32
        [batch][queries][n_q_heads], or None."""
        if getattr(q, "ndim", 0) != 4:
            raise TypeError("q must be a CUDA (HIP) tensor [batch][queries][n_q_heads][head_dim]")
        B, n = int(q.shape[0]), int(q.shape[1])
        shape = (B, n, self.n_q_heads, self.head_dim)
        qp, op = self._tensor(q, shape, "q"), self._tensor(out, shape, "out")
        tp, width = self._table(table, B)
        _check(self.lib.raas_quant_attention(self._h, layer, qp, tp, width, self._lengths(lens, B, "lens"),
                                             self._ints(counts, (B,), "counts"), B, n, op,
                                             self._floats(lse, shape[:3], "lse"), _stream(stream, self.device)),
               "raas_quant_attention")

    def prepare_step(self, layer: int, q, k_new, v_new, out, table, lens, lse=None, k_held=None, v_held=None,
                     prefix=None, stream=None) -> PreparedQuantStep:
        """Checks and converts the arguments of one raas_quant_step call once, so a
        loop can replay them with decode_prepared(). q, out: [batch][n_q_heads]
        [head_dim]; k_new, v_new, and optionally k_held, v_held: [batch][n_kv_heads]
        [head_dim]; table: int32 [batch][width]; lens: int32 [batch], the tokens held
        so far; lse: fp32 [batch][n_q_heads], or None; prefix: a SharedPrefix, or None."""
        if prefix is not None and not isinstance(prefix, SharedPrefix):
            raise TypeError("prefix must be a SharedPrefix")
        if getattr(q, "ndim", 0) != 3:
            raise TypeError("q must be a CUDA (HIP) tensor [batch][n_q_heads][head_dim]")
        B = int(q.shape[0])
        rows, tokens = (B, self.n_q_heads, self.head_dim), (B, self.n_kv_heads, self.head_dim)
        tp, width = self._table(table, B)
        step = PreparedQuantStep((
            self._h, layer,
            self._tensor(q, rows, "q"),
            self._tensor(k_new, tokens, "k_new"),
            self._tensor(v_new, tokens, "v_new"),
            tp, width, self._lengths(lens, B, "lens"), B,
            self._tensor(out, rows, "out"),
            self._floats(lse, rows[:2], "lse"),
            self._tensor(k_held, tokens, "k_held", optional=True),
            self._tensor(v_held, tokens, "v_held", optional=True),
            None if prefix is None else prefix.handle,
            _stream(stream, self.device),
        ))
        step.prefix = prefix
        step.tensors = (q, k_new, v_new, table, lens, out, lse, k_held, v_held)
        return step

    def decode_prepared(self, step: PreparedQuantStep):
        if step.prefix is not None and not step.prefix.handle.value:
            raise ValueError("the step's prefix is closed")
        _check(self.lib.raas_quant_step(*step), "raas_quant_step")

    def decode_step(self, layer: int, q, k_new, v_new, out, table, lens, lse=None, k_held=None, v_held=None, prefix=None,
                    stream=None):
        """One decode step of one layer (raas_quant_step)."""
        self.decode_prepared(self.prepare_step(layer, q, k_new, v_new, out, table, lens, lse, k_held, v_held, prefix,
                                               stream))

    def device_bytes(self) -> int:
        return int(self.lib.raas_quant_cache_bytes(self._h))
