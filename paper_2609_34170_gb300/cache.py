"""ContextCache: keys and values of a VLM's layers in 8 bits, the attention that
reads them, and eviction by attention mass (the C ABI of include/ravel_cache.h).

A robot's prompt goes in layer by layer (``append``, ``attend``), then its
decoded tokens one by one; ``evict`` shrinks what is held to a budget, and
``read`` returns it in the layout of a layer of ``RollingSession.set_context``.
Positions, lengths and counts are int32 CUDA tensors with one entry per robot.
Every call is enqueued on ``stream`` (None: the current one of the cache's device).

The calls look their arguments over and hand addresses to the library, nothing
else: at one token the host takes as long as the GPU.
"""
from __future__ import annotations

from . import _binding as B


class ContextCache:
    def __init__(self, layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, max_tokens: int, max_batch: int = 1,
                 max_queries: int = 1, dtype: str = "bf16", device: int = 0):
        """Room for max_tokens tokens of max_batch robots; max_queries: the most
        queries per robot in one ``attend``; dtype ("bf16" or "fp32"): that of
        the tensors that go in and come out."""
        import torch
        if dtype not in ("bf16", "fp32"):
            raise ValueError(f"dtype must be 'bf16' or 'fp32', got {dtype!r}")
        self.torch = torch
        self.layers, self.n_q_heads, self.n_kv_heads, self.head_dim = layers, n_q_heads, n_kv_heads, head_dim
        self.max_tokens, self.max_batch, self.max_queries = max_tokens, max_batch, max_queries
        self.device = torch.device("cuda", device)
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.handle = B.ravel_cache_create(layers, n_q_heads, n_kv_heads, head_dim, max_tokens, max_batch, max_queries,
                                           B.RAVEL_BF16 if dtype == "bf16" else B.RAVEL_FP32, device)
        self._lib = B.load()
        arguments = self.handle.arguments
        self._rows, self._ints, self._mass, self._dense = arguments.rows, arguments.ints, arguments.mass, arguments.dense
        self._int32, self._float32 = torch.int32, torch.float32
        self._index, self._current_stream = self.device.index, B.current_stream_getter()

    # -- arguments
    def _stream(self, stream):
        if stream is None:
            return self._current_stream(self._index)
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)

    def _empty(self, shape, dtype, stream, zeros=False):
        """A new tensor of the stream that is going to write it."""
        if stream is None:
            return (self.torch.zeros if zeros else self.torch.empty)(shape, dtype=dtype, device=self.device)
        return B.new_tensor(shape, dtype, self.device, stream, zeros)

    # -- calls
    def append(self, layer: int, k, v, starts=None, counts=None, stream=None):
        """Store tokens k, v [B, n, Hkv, hd]: token i < counts[b] of robot b at
        position starts[b] + i (None: all n of them; from position 0)."""
        strides = self._rows(k, self.n_kv_heads, "k")
        shape = k.shape
        if v.shape != shape or self._rows(v, self.n_kv_heads, "v") != strides:
            raise ValueError("k and v must have the same shape and strides")
        batch, n = shape[0], shape[1]
        status = self._lib.ravel_cache_append(self.handle, layer, batch, n, k.data_ptr(), v.data_ptr(), strides[0], strides[1],
                                              self._ints(starts, batch, "starts"), self._ints(counts, batch, "counts"),
                                              self._stream(stream))
        if status:
            B._check_cache(self.handle, status, "ravel_cache_append")

    def append_rotary(self, layer: int, rotary, q, k, v, starts=None, counts=None, positions=None, q_out=None, stream=None):
        """``append`` of keys turned by a ``Rotary`` to their positions (int32 [B, n]; None:
        starts[b] + i), and the queries q [B, n, Hq, hd] turned with them: returned, or written to
        q_out, which may be q itself (rows from counts[b] on are not written; of a new tensor they are
        zeros).  q None: keys alone."""
        r = rotary.handle
        if getattr(r, "rotary", None) is None:
            raise ValueError("rotary must be an open Rotary")
        rows, ints = self._rows, self._ints
        shape = k.shape
        krs, kts = rows(k, self.n_kv_heads, "k")
        if v.shape != shape:
            raise ValueError("k and v must have the same shape")
        vrs, vts = rows(v, self.n_kv_heads, "v")
        batch, n = shape[0], shape[1]
        if (layer | batch | n) >> 31:
            B._fit_ints("append_rotary", layer, batch, n)
        q_at = out_at = None
        qrs = qts = ors = ots = 0
        if q is not None:
            qrs, qts = rows(q, self.n_q_heads, "q")
            shape = q.shape
            if shape[0] != batch or shape[1] != n:
                raise ValueError("q must have as many tokens as k")
            if q_out is None:
                q_out = self._empty(shape, q.dtype, stream, zeros=counts is not None)
            elif q_out.shape != shape:
                raise ValueError("q_out must have q's shape")
            if q_out is q:
                ors, ots = qrs, qts
            else:
                ors, ots = rows(q_out, self.n_q_heads, "q_out")
            q_at, out_at = q.data_ptr(), q_out.data_ptr()
        elif q_out is not None:
            raise ValueError("q and q_out go together")
        status = self._lib.ravel_cache_append_rotary(
            self.handle, layer, r, batch, n, q_at, qrs, qts, out_at, ors, ots, k.data_ptr(), krs, kts, v.data_ptr(), vrs, vts,
            ints(starts, batch, "starts"), self._dense(positions, (batch, n), self._int32, "positions") if positions is not None else None,
            ints(counts, batch, "counts"), self._stream(stream))
        if status:
            B._check_cache(self.handle, status, "ravel_cache_append_rotary")
        return q_out

    def attend(self, layer: int, q, lengths, counts=None, causal: bool = True, window: int = 0, sinks: int = 0,
               scale: float = 0.0, max_length: int | None = None, out=None, mass=None, add_mass: bool = False, stream=None):
        """softmax(scale q k) v of queries q [B, n, Hq, hd] over robot b's
        lengths[b] tokens, its counts[b] queries being the last ones (None: n);
        causal: query i sees up to its own position, with `window` the last
        `window` of those and the first `sinks`.  mass (float32 [B, Hkv, tokens]):
        receives, or with add_mass is increased by, the attention mass that each
        token drew.  max_length: a bound of the lengths (None: the cache's
        room).  Launches are planned for it, so that a bound near the lengths is
        worth giving: one token over 816 takes 8 us with it, 39 in a cache with
        room for 8192 without."""
        qr, qt = self._rows(q, self.n_q_heads, "q")
        shape = q.shape
        batch, n = shape[0], shape[1]
        if out is None:
            out = self._empty(shape, q.dtype, stream)
        elif out.shape != shape:
            raise ValueError("out must have q's shape")
        if out.dtype is q.dtype and out.stride() == q.stride() and out.get_device() == self._index:
            outr, outt = qr, qt
        else:
            outr, outt = self._rows(out, self.n_q_heads, "out")
        if lengths is None:
            raise ValueError("lengths must be given")
        mass_at, mass_len = self._mass(mass, batch) if mass is not None else (None, 0)
        status = self._lib.ravel_cache_attend(
            self.handle, layer, batch, n, q.data_ptr(), qr, qt, out.data_ptr(), outr, outt,
            self._ints(lengths, batch, "lengths"), self._ints(counts, batch, "counts"),
            self.max_tokens if max_length is None else max_length, 1 if causal else 0, window, sinks, scale, mass_at, mass_len,
            1 if add_mass else 0, self._stream(stream))
        if status:
            B._check_cache(self.handle, status, "ravel_cache_attend")
        return out

    def evict(self, layer: int, to: "ContextCache", to_layer: int, lengths, mass, keep: int, sinks: int = 0,
              recent: int = 0, stream=None):
        """Of every robot and KV head the `keep` tokens that stay go into layer
        to_layer of `to`: the first `sinks`, the last `recent`, and the heaviest
        of the rest by mass [B, Hkv, tokens].  Returns their number per robot
        [B], their positions [B, Hkv, keep] (then -1) and their mass (then 0)."""
        mass_at, mass_len = self._mass(mass, None)
        batch = mass.shape[0]
        new_lengths = self._empty((batch,), self._int32, stream)
        shape = (batch, self.n_kv_heads, max(keep, 1))
        index, new_mass = self._empty(shape, self._int32, stream), self._empty(shape, self._float32, stream)
        status = self._lib.ravel_cache_evict(self.handle, layer, to.handle, to_layer, batch, self._ints(lengths, batch, "lengths"),
                                             mass_at, mass_len, keep, sinks, recent, new_lengths.data_ptr(), index.data_ptr(),
                                             new_mass.data_ptr(), self._stream(stream))
        if status:
            B._check_cache(self.handle, status, "ravel_cache_evict")
        return new_lengths, index, new_mass

    def read(self, layer: int, batch: int, n: int, firsts=None, lengths=None, stream=None):
        """The values held of n tokens per robot from position firsts[b] on
        (None: 0), zeros from lengths[b] on: k, v [B, Hkv, n, hd]."""
        shape = (batch, self.n_kv_heads, n, self.head_dim)
        k, v = self._empty(shape, self.dtype, stream), self._empty(shape, self.dtype, stream)
        status = self._lib.ravel_cache_read(self.handle, layer, batch, n, self._ints(firsts, batch, "firsts"),
                                            self._ints(lengths, batch, "lengths"), k.data_ptr(), v.data_ptr(),
                                            self._stream(stream))
        if status:
            B._check_cache(self.handle, status, "ravel_cache_read")
        return k, v

    def reset(self):
        """Clear a device error (lengths or positions out of range); what is held stays."""
        B.ravel_cache_reset(self.handle)

    def close(self):
        if getattr(self, "handle", None) is not None:
            B.ravel_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
