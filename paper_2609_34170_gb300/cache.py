"""ContextCache: keys and values of a VLM's layers in 8 bits, the attention that
reads them, and eviction by attention mass (the C ABI of include/ravel_cache.h).

A robot's prompt goes in layer by layer (``append``, ``attend``), then its
decoded tokens one by one; ``evict`` shrinks what is held to a budget, and
``read`` returns it in the layout of a layer of ``RollingSession.set_context``.
Positions, lengths and counts are int32 CUDA tensors with one entry per robot.
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

    def _of_dtype(self, t, heads, name):
        if t.dtype != self.dtype or t.dim() != 4 or t.shape[2] != heads or t.shape[3] != self.head_dim:
            raise ValueError(f"{name} must be [batch, n, {heads}, {self.head_dim}] of dtype {self.dtype}, "
                             f"got {tuple(t.shape)} of {t.dtype}")

    def _empty(self, shape, dtype, stream):
        """A new tensor of the stream that is going to write it."""
        t = self.torch
        if stream is None:
            return t.empty(shape, dtype=dtype, device=self.device)
        if not hasattr(stream, "cuda_stream"):
            stream = t.cuda.ExternalStream(int(stream), device=self.device)
        with t.cuda.stream(stream):
            return t.empty(shape, dtype=dtype, device=self.device)

    def append(self, layer: int, k, v, starts=None, counts=None, stream=None):
        """Store tokens k, v [B, n, Hkv, hd]: token i < counts[b] of robot b at
        position starts[b] + i (None: all n of them; from position 0)."""
        self._of_dtype(k, self.n_kv_heads, "k")
        B.ravel_cache_append(self.handle, layer, k, v, starts, counts, stream)

    def attend(self, layer: int, q, lengths, counts=None, causal: bool = True, window: int = 0, sinks: int = 0,
               scale: float = 0.0, max_length: int | None = None, out=None, mass=None, add_mass: bool = False, stream=None):
        """softmax(scale q k) v of queries q [B, n, Hq, hd] over robot b's
        lengths[b] tokens, its counts[b] queries being the last ones (None: n);
        causal: query i sees up to its own position, with `window` the last
        `window` of those and the first `sinks`.  mass (float32 [B, Hkv, tokens]):
        receives, or with add_mass is increased by, the attention mass that each
        token drew.  max_length: a bound of the lengths, if one below the
        cache's (or mass's) room is known; launches are planned for it."""
        self._of_dtype(q, self.n_q_heads, "q")
        if max_length is None:
            max_length = self.max_tokens
        if mass is not None:
            if mass.dim() != 3 or mass.shape[:2] != (q.shape[0], self.n_kv_heads):
                raise ValueError(f"mass must be [{q.shape[0]}, {self.n_kv_heads}, tokens], got {tuple(mass.shape)}")
        if out is None:
            out = self._empty(q.shape, q.dtype, stream)
        B.ravel_cache_attend(self.handle, layer, q, out, lengths, counts, max_length, causal, window, sinks, scale, mass,
                             add_mass, stream)
        return out

    def evict(self, layer: int, to: "ContextCache", to_layer: int, lengths, mass, keep: int, sinks: int = 0,
              recent: int = 0, stream=None):
        """Of every robot and KV head the `keep` tokens that stay go into layer
        to_layer of `to`: the first `sinks`, the last `recent`, and the heaviest
        of the rest by mass [B, Hkv, tokens].  Returns their number per robot
        [B], their positions [B, Hkv, keep] (then -1) and their mass (then 0)."""
        t = self.torch
        if mass.dim() != 3 or mass.shape[1] != self.n_kv_heads:
            raise ValueError(f"mass must be [batch, {self.n_kv_heads}, tokens], got {tuple(mass.shape)}")
        batch = mass.shape[0]
        new_lengths = self._empty((batch,), t.int32, stream)
        index = self._empty((batch, self.n_kv_heads, max(keep, 1)), t.int32, stream)
        new_mass = self._empty(index.shape, t.float32, stream)
        B.ravel_cache_evict(self.handle, layer, to.handle, to_layer, lengths, mass, keep, sinks, recent, new_lengths, index,
                            new_mass, stream)
        return new_lengths, index, new_mass

    def read(self, layer: int, batch: int, n: int, firsts=None, lengths=None, stream=None):
        """The values held of n tokens per robot from position firsts[b] on
        (None: 0), zeros from lengths[b] on: k, v [B, Hkv, n, hd]."""
        k, v = (self._empty((batch, self.n_kv_heads, n, self.head_dim), self.dtype, stream) for _ in "kv")
        B.ravel_cache_read(self.handle, layer, k, v, firsts, lengths, stream)
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
