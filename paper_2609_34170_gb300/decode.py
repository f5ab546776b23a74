"""What a VLM's decode step needs beside the ContextCache (the C ABI of
include/ravel_decode.h): rotary positions, products of few rows with 4-bit
weights, and drawing a token from logits.

A decoded token's way: ``Weights4.product`` to queries, keys and values,
``ContextCache.append_rotary`` and ``attend``, products again, and
``draw_tokens`` from the logits.  Every call is enqueued on ``stream`` (None:
the current one of the tensors' device).
"""
from __future__ import annotations

from . import _binding as B


def _current_stream(device: int) -> int:
    """Address of a device's current stream."""
    global _current_stream
    _current_stream = B.current_stream_getter()
    return _current_stream(device)


class _Handle:
    """Owns a handle of the library on one device."""

    def _open(self, handle, device: int):
        import torch
        self.handle = handle
        self.device = torch.device("cuda", device)
        self._index, self._current_stream = device, B.current_stream_getter()

    def _stream(self, stream):
        if stream is None:
            return self._current_stream(self._index)
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)

    def close(self):
        if getattr(self, "handle", None) is not None:
            self._destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Rotary(_Handle):
    """Turns pairs of a head's first `dims` dims, (i, i + dims / 2) or interleaved (2i, 2i + 1), by
    the angle position * f_i, f_i = base^(-2i / dims).  For contexts longer than a model was trained
    on, frequencies are divided by `factor`: all of them, or, with an original_length, in full those
    that make at most `low` turns over it, not those that make `high` or more, and in between in
    proportion (to those turns; for tables that go by the dims' index, give frequencies).  amplitude scales
    what is turned; frequencies [dims / 2] replaces the f_i."""
    _destroy = staticmethod(B.ravel_rotary_destroy)

    def __init__(self, dims: int, base: float = 10000.0, interleaved: bool = False, factor: float = 1.0,
                 original_length: float = 0.0, low: float = 1.0, high: float = 32.0, amplitude: float = 1.0,
                 frequencies=None, device: int = 0):
        self.dims = dims
        self._open(B.ravel_rotary_create(dims, base, interleaved, factor, original_length, low, high, amplitude, frequencies,
                                         device), device)

    def apply(self, x, starts=None, counts=None, positions=None, out=None, stream=None):
        """x [B, n, heads, head_dim] (heads of a token contiguous: query and key columns of a projection
        are one call) turned to positions starts[b] + i (None: i) or positions [B, n], int32.  out may
        be x itself; tokens from counts[b] on are not written (of a new tensor they are zeros).
        The transpose, which is the gradient, is the rotation to the positions' negatives."""
        if out is None:
            out = B.new_tensor(x.shape, x.dtype, self.device, stream, zeros=counts is not None)
        B.ravel_rotary_apply(self.handle, x, out, starts, positions, counts, self._stream(stream))
        return out


class Weights4(_Handle):
    """A matrix [n, k] of 4-bit weights (c - z) s, with a zero point and a bf16 scale per
    `group` (32, 64 or 128) ks of a row.  (fp16 scales rounded to bf16 move by up to 2^-8 of their size.)"""
    _destroy = staticmethod(B.ravel_w4_destroy)

    def __init__(self, n: int, k: int, group: int = 128, device: int = 0):
        self.n, self.k, self.group = n, k, group
        self._open(B.ravel_w4_create(n, k, group, device), device)

    @classmethod
    def quantize(cls, w, group: int = 128, stream=None):
        """Of a matrix w [n, k] (bf16 or fp32) its nearest codes."""
        made = cls(w.shape[0], w.shape[1], group, w.get_device())
        made.load(*quantize4(w, group, stream), stream=stream)
        return made

    def load(self, codes, scales, zeros, stream=None):
        """codes uint8 [n, (k + 1) // 2] (even k in the low nibble), scales bf16 and zeros uint8
        [n, groups].  Waits for the stream; no product may be running."""
        B.ravel_w4_load(self.handle, codes, scales, zeros, self._stream(stream))

    def reset(self):
        """Clear a device error (a bounded wait that ran out)."""
        B.ravel_w4_reset(self.handle)

    def read(self, dtype=None, out=None, stream=None):
        """The weights held, [n, k] in bf16 or fp32, for example for products of whole prompts."""
        if out is None:
            import torch
            out = B.new_tensor((self.n, self.k), dtype or torch.bfloat16, self.device, stream)
        B.ravel_w4_read(self.handle, out, self._stream(stream))
        return out

    def product(self, x, out=None, epi: str = "store", bias=None, dtype=None, stream=None):
        """x [m, k] (bf16) times the rows, plus bias [n] (fp32), by epilogue: "store", "silu", "add" (out,
        fp32, is increased) or "geglu" (rows in blocks of 64 gate rows and their 64 up rows).  A new out
        is of dtype (bf16)."""
        code = B.W4_EPILOGUES.get(epi)
        if code is None:
            raise ValueError(f"epi must be one of {sorted(B.W4_EPILOGUES)}, got {epi!r}")
        if out is None:
            if code == 2:
                raise ValueError("epi 'add' needs an out to add to")
            import torch
            out = B.new_tensor((x.shape[0], self.n // 2 if code == 3 else self.n), dtype or torch.bfloat16, self.device, stream)
        B.ravel_w4_gemm(self.handle, x, code, out, bias, self._stream(stream))
        return out


def quantize4(w, group: int = 128, stream=None):
    """Nearest 4-bit codes of w [n, k]: codes uint8 [n, (k + 1) // 2], scales bf16 and zeros uint8
    [n, groups], as ``Weights4.load`` takes them."""
    import torch
    if w.dim() != 2 or w.get_device() < 0 or group not in (32, 64, 128):
        raise ValueError(f"w must be a CUDA tensor [n, k] and group 32, 64 or 128, got {tuple(w.shape)} on {w.device} and {group}")
    n, k = w.shape
    groups = -(-k // group)
    codes = B.new_tensor((n, (k + 1) // 2), torch.uint8, w.device, stream)
    scales, zeros = (B.new_tensor((n, groups), t, w.device, stream) for t in (torch.bfloat16, torch.uint8))
    if stream is None:
        stream = _current_stream(w.get_device())
    B.ravel_w4_quantize(w, group, codes, scales, zeros, stream)
    return codes, scales, zeros


def draw_tokens(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, log_probs: bool = False, tokens=None, stream=None):
    """Of each row of logits [B, vocab] a token (int32 [B]) by given random numbers u (fp32 [B], 0 <= u
    < 1), and with log_probs its log-probability.  temperature, top_p, min_p (fp32 [B]) and top_k (int32
    [B]) are settings of each row or None; see ravel_decode.h for their order and what they leave.  A row that
    cannot be drawn from (nothing but -inf, a NaN, a setting out of range) gives -1."""
    types = B._types()
    index = logits.get_device()
    if index < 0:
        raise ValueError(f"logits must be a CUDA tensor, got one on {logits.device}")
    shape, device = (logits.shape[0],), logits.device
    if tokens is None:
        tokens = B.new_tensor(shape, types.i32, device, stream)
    logs = B.new_tensor(shape, types.f32, device, stream) if log_probs else None
    if stream is None:
        stream = _current_stream(index)
    B.ravel_draw_tokens(logits, u, temperature, top_k, top_p, min_p, tokens, logs, stream)
    return (tokens, logs) if log_probs else tokens
