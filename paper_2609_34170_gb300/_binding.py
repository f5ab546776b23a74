"""ctypes binding of libravel: the C ABI of include/ravel.h, same names, with
argument marshalling only (every step of the path runs in the CUDA kernels).

The library must have been built (``paper_2609_34170_gb300.build.build()``);
there is no fallback: a missing library raises on first use.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

from . import build as _build

RAVEL_FP32, RAVEL_BF16 = 0, 1
RAVEL_MASK_FULL, RAVEL_MASK_SLOT_ISOLATED = 0, 1
RAVEL_FAULT_PREFIX_LEN, RAVEL_FAULT_WITHHOLD_ARRIVAL = 1, 2

STATUS = ["RAVEL_OK", "RAVEL_EINVAL", "RAVEL_ESHAPE", "RAVEL_ENOMEM", "RAVEL_ECUDA", "RAVEL_ENOCONTEXT",
          "RAVEL_EBUSY", "RAVEL_EDEVICE", "RAVEL_ETIMEOUT", "RAVEL_ENOTREADY"]


class RavelConfig(C.Structure):
    _fields_ = [(n, C.c_int) for n in (
        "layers", "width", "n_q_heads", "n_kv_heads", "head_dim", "mlp_dim", "slots", "action_dim",
        "max_prefix", "fop_tokens", "max_batch", "dtype", "mask_mode", "fop_adapter_every", "per_robot_times")]


WEIGHT_FIELDS = ("t_w1", "t_b1", "t_w2", "t_b2", "d_w1", "d_b1", "d_w2", "d_b2", "mod_w", "mod_b",
                 "in_w", "in_b", "fop_gamma", "w_qkv", "w_o", "w_gate", "w_up", "w_down", "out_w", "out_b")


ADAPTER_FIELDS = ("a_gamma", "a_zgamma", "a_wq", "a_wkv", "a_wo", "a_gate")


class RavelWeights(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in WEIGHT_FIELDS] + [("on_device", C.c_int)]
                + [(n, C.c_void_p) for n in ADAPTER_FIELDS])


class RavelCacheConfig(C.Structure):
    _fields_ = [(n, C.c_int) for n in (
        "layers", "n_q_heads", "n_kv_heads", "head_dim", "max_tokens", "max_batch", "max_queries", "dtype")]


class RavelRotaryConfig(C.Structure):
    _fields_ = ([("dims", C.c_int), ("interleaved", C.c_int)]
                + [(n, C.c_double) for n in ("base", "factor", "original_length", "low", "high", "amplitude")]
                + [("frequencies", C.POINTER(C.c_double))])


class RavelError(RuntimeError):
    def __init__(self, status: int, msg: str):
        self.status = status
        name = STATUS[status] if 0 <= status < len(STATUS) else str(status)
        super().__init__(f"{name}: {msg}")


_lib = None


def lib_path() -> str:
    return _build.LIB


def load(path: str | None = None):
    """Load libravel.so (once).  Raises OSError if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or lib_path()
    if not os.path.exists(path):
        raise OSError(f"{path} is missing: build it with paper_2609_34170_gb300.build.build()")
    L = C.CDLL(path)
    vp, i, ll, pp = C.c_void_p, C.c_int, C.c_longlong, C.POINTER(C.c_void_p)
    sig = {
        "ravel_create": (i, [C.POINTER(RavelConfig), C.POINTER(RavelWeights), i, pp]),
        "ravel_destroy": (None, [vp]),
        "ravel_reset": (i, [vp, i, vp, vp, vp]),
        "ravel_set_context": (i, [vp, vp, vp, i, vp]),
        "ravel_set_context_robots": (i, [vp, vp, i, vp, vp, i, vp]),
        "ravel_roll_step": (i, [vp, vp, vp, vp, vp, vp, vp, vp]),
        "ravel_denoise_chunk": (i, [vp, vp, i, vp, vp, vp, vp]),
        "ravel_roll_step_rel": (i, [vp, vp, vp, vp, vp, vp, vp, vp, vp]),
        "ravel_set_relative_dims": (i, [vp, vp]),
        "ravel_copy_inputs": (i, [vp, i, vp, vp, vp, vp]),
        "ravel_get_state": (i, [vp, vp]),
        "ravel_set_state": (i, [vp, vp]),
        "ravel_step_kernel_count": (i, [vp]),
        "ravel_profile_step": (i, [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i, vp]),
        "ravel_kernel_kind_name": (C.c_char_p, [i]),
        "ravel_gemm": (i, [vp, vp, i, i, i, vp, i, i, i, vp, i, i, vp, vp]),
        "ravel_gemm_noalloc": (i, [vp, i, i, i, vp, i, i, i, vp, i, i, vp, vp]),
        "ravel_gemm_noalloc_status": (i, [vp]),
        "ravel_debug_inject": (i, [vp, i, i, vp]),
        "ravel_status_string": (C.c_char_p, [i]),
        "ravel_last_error": (C.c_char_p, [vp]),
        "ravel_cache_create": (i, [C.POINTER(RavelCacheConfig), i, pp]),
        "ravel_cache_destroy": (None, [vp]),
        "ravel_cache_reset": (i, [vp]),
        "ravel_cache_append": (i, [vp, i, i, i, vp, vp, ll, ll, vp, vp, vp]),
        "ravel_cache_attend": (i, [vp, i, i, i, vp, ll, ll, vp, ll, ll, vp, vp, i, i, i, i, C.c_float, vp, ll, i, vp]),
        "ravel_cache_evict": (i, [vp, i, vp, i, i, vp, vp, ll, i, i, i, vp, vp, vp, vp]),
        "ravel_cache_read": (i, [vp, i, i, i, vp, vp, vp, vp, vp]),
        "ravel_cache_last_error": (C.c_char_p, [vp]),
        "ravel_rotary_create": (i, [C.POINTER(RavelRotaryConfig), i, pp]),
        "ravel_rotary_destroy": (None, [vp]),
        "ravel_rotary_apply": (i, [vp, i, i, i, i, i, vp, ll, ll, vp, ll, ll, vp, vp, vp, vp]),
        "ravel_cache_append_rotary": (i, [vp, i, vp, i, i, vp, ll, ll, vp, ll, ll, vp, ll, ll, vp, ll, ll, vp, vp, vp, vp]),
        "ravel_w4_create": (i, [i, i, i, i, pp]),
        "ravel_w4_destroy": (None, [vp]),
        "ravel_w4_reset": (i, [vp]),
        "ravel_w4_load": (i, [vp, vp, vp, vp, vp]),
        "ravel_w4_quantize": (i, [vp, i, i, i, i, i, vp, vp, vp, vp]),
        "ravel_w4_read": (i, [vp, vp, i, i, vp]),
        "ravel_w4_gemm": (i, [vp, vp, i, i, i, vp, i, i, vp, vp]),
        "ravel_draw_tokens": (i, [vp, i, i, ll, i, vp, vp, vp, vp, vp, vp, vp, vp]),
        "ravel_decode_last_error": (C.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype, f.argtypes = res, args
    _lib = L
    return L


def _check(h, status: int, what: str):
    if status != 0:
        msg = load().ravel_last_error(h).decode() if h else ""
        raise RavelError(status, f"{what}: {msg}")


def _dptr(t, dtype=None, name="tensor"):
    """Device pointer of a contiguous CUDA tensor (or None)."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream_ptr(stream):
    if type(stream) is int:
        return stream
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def ravel_create(cfg, weights: dict, device: int = 0, max_batch: int | None = None,
                 max_prefix: int | None = None, mask_mode: int = RAVEL_MASK_FULL):
    """cfg: an object with the ExpertConfig fields; weights: name -> float32
    array in math layout (numpy host arrays or CUDA tensors, not mixed)."""
    L = load()
    c = RavelConfig(cfg.layers, cfg.width, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.mlp_dim, cfg.slots,
                    cfg.action_dim, max_prefix or cfg.prefix, cfg.fop_tokens, max_batch or cfg.batch,
                    RAVEL_BF16 if cfg.dtype == "bf16" else RAVEL_FP32, mask_mode,
                    getattr(cfg, "fop_adapter_every", 0), getattr(cfg, "per_robot_times", 0))
    on_dev = None
    keep = []
    w = RavelWeights()
    for n in WEIGHT_FIELDS + ADAPTER_FIELDS:
        if n not in weights:   # adapter tensors of a network without adapters
            continue
        a = weights[n]
        if isinstance(a, np.ndarray):
            a = np.ascontiguousarray(a, dtype=np.float32)
            keep.append(a)
            ptr, dev = a.ctypes.data, False
        else:
            ptr, dev = _dptr(a, name=n), True
            keep.append(a)
        if on_dev is None:
            on_dev = dev
        elif on_dev != dev:
            raise ValueError("weights must be all host arrays or all CUDA tensors")
        setattr(w, n, ptr)
    w.on_device = int(bool(on_dev))
    h = C.c_void_p()
    st = L.ravel_create(C.byref(c), C.byref(w), device, C.byref(h))
    if st != 0:
        raise RavelError(st, "ravel_create failed (see stderr)")
    return h


def ravel_destroy(h):
    load().ravel_destroy(h)


def ravel_reset(h, batch: int, seeds, buffer, stream=None):
    seeds = np.ascontiguousarray(seeds, dtype=np.uint64)
    import torch
    _check(h, load().ravel_reset(h, batch, seeds.ctypes.data, _dptr(buffer, torch.float32, "buffer"),
                                 _stream_ptr(stream)), "ravel_reset")


def ravel_set_context(h, k, v, prefix_len: int, side_stream=None):
    _check(h, load().ravel_set_context(h, _dptr(k, name="k"), _dptr(v, name="v"), prefix_len,
                                       _stream_ptr(side_stream)), "ravel_set_context")


def ravel_set_context_robots(h, robots, k, v, prefix_len: int, side_stream=None):
    """New contexts for the listed robots only (k, v [L, len(robots), Hkv, prefix_len, hd])."""
    idx = np.ascontiguousarray(np.asarray(robots, dtype=np.int32))
    _check(h, load().ravel_set_context_robots(h, idx.ctypes.data, int(idx.size), _dptr(k, name="k"), _dptr(v, name="v"),
                                              prefix_len, _stream_ptr(side_stream)), "ravel_set_context_robots")


def ravel_roll_step(h, buffer, slot_times, obs_tokens, delta, released, velocity=None, stream=None):
    import torch
    f32 = torch.float32
    _check(h, load().ravel_roll_step(
        h, _dptr(buffer, f32, "buffer"), _dptr(slot_times, f32, "slot_times"), _dptr(obs_tokens, name="obs_tokens"),
        _dptr(delta, f32, "delta"), _dptr(released, f32, "released"), _dptr(velocity, f32, "velocity"),
        _stream_ptr(stream)), "ravel_roll_step")


def ravel_roll_step_rel(h, buffer, slot_times, obs_tokens, delta, state, released, velocity=None, stream=None):
    import torch
    f32 = torch.float32
    _check(h, load().ravel_roll_step_rel(
        h, _dptr(buffer, f32, "buffer"), _dptr(slot_times, f32, "slot_times"), _dptr(obs_tokens, name="obs_tokens"),
        _dptr(delta, f32, "delta"), _dptr(state, f32, "state"), _dptr(released, f32, "released"),
        _dptr(velocity, f32, "velocity"), _stream_ptr(stream)), "ravel_roll_step_rel")


def ravel_set_relative_dims(h, mask):
    m = np.ascontiguousarray(mask, dtype=np.float32)
    _check(h, load().ravel_set_relative_dims(h, m.ctypes.data), "ravel_set_relative_dims")


def ravel_denoise_chunk(h, chunk, n_steps: int, obs_tokens, delta, velocity=None, stream=None):
    import torch
    f32 = torch.float32
    _check(h, load().ravel_denoise_chunk(h, _dptr(chunk, f32, "chunk"), n_steps, _dptr(obs_tokens, name="obs_tokens"),
                                         _dptr(delta, f32, "delta"), _dptr(velocity, f32, "velocity"),
                                         _stream_ptr(stream)), "ravel_denoise_chunk")


def ravel_profile_step(h, buffer, slot_times, obs_tokens, delta, released, velocity=None, stream=None,
                       cap: int = 4096):
    """Eager step with per-launch timing: returns [(kind_name, ms), ...]."""
    import torch
    f32 = torch.float32
    ms = np.zeros(cap, np.float32)
    kinds = np.zeros(cap, np.int32)
    n = C.c_int(0)
    _check(h, load().ravel_profile_step(
        h, _dptr(buffer, f32, "buffer"), _dptr(slot_times, f32, "slot_times"), _dptr(obs_tokens, name="obs_tokens"),
        _dptr(delta, f32, "delta"), _dptr(released, f32, "released"), _dptr(velocity, f32, "velocity"),
        _stream_ptr(stream), ms.ctypes.data, kinds.ctypes.data, cap, C.byref(n)), "ravel_profile_step")
    k = min(n.value, cap)
    return [(load().ravel_kernel_kind_name(int(kinds[i])).decode(), float(ms[i])) for i in range(k)]


def ravel_gemm(h, X, W, epi: int, out, bias=None, K: int | None = None, stream=None):
    """out (op)= X[:, :K] @ W[:, :K]^T (+ bias) on the device; see ravel.h."""
    import torch
    M, lda = X.shape
    N, ldw = W.shape
    K = lda if K is None else K
    od = 1 if out.dtype == torch.bfloat16 else 0
    _check(h, load().ravel_gemm(h, _dptr(X, name="X"), M, K, lda, _dptr(W, name="W"), N, ldw, epi,
                                _dptr(out, name="out"), out.shape[1], od, _dptr(bias, torch.float32, "bias"),
                                _stream_ptr(stream)), "ravel_gemm")


def ravel_gemm_noalloc(X, W, epi: int, out, bias=None, K: int | None = None, stream=None):
    """ravel_gemm without a handle and without device allocation (see ravel.h)."""
    import torch
    M, lda = X.shape
    N, ldw = W.shape
    K = lda if K is None else K
    od = 1 if out.dtype == torch.bfloat16 else 0
    _check(None, load().ravel_gemm_noalloc(_dptr(X, torch.bfloat16, "X"), M, K, lda, _dptr(W, torch.bfloat16, "W"),
                                           N, ldw, epi, _dptr(out, name="out"), out.shape[1], od,
                                           _dptr(bias, torch.float32, "bias"), _stream_ptr(stream)),
           "ravel_gemm_noalloc")


def ravel_gemm_noalloc_status(stream=None) -> int:
    """Status of the allocation-free GEMM's device error word (read and
    cleared); returned as the raw ravel_status value."""
    return int(load().ravel_gemm_noalloc_status(_stream_ptr(stream)))


def ravel_debug_inject(h, fault: int, count: int = 1, stream=None):
    """Fault injection of the failure-path tests (see ravel.h)."""
    _check(h, load().ravel_debug_inject(h, fault, count, _stream_ptr(stream)), "ravel_debug_inject")


def ravel_copy_inputs(h, n: int, dst, src, nbytes, stream=None):
    """dst[i] <- src[i] for n device arrays in one launch: ctypes arrays of
    addresses (c_void_p) and sizes (c_size_t)."""
    _check(h, load().ravel_copy_inputs(h, n, dst, src, nbytes, _stream_ptr(stream)), "ravel_copy_inputs")


def ravel_get_state(h, batch: int) -> np.ndarray:
    out = np.zeros(batch, dtype=np.uint64)
    _check(h, load().ravel_get_state(h, out.ctypes.data), "ravel_get_state")
    return out


def ravel_set_state(h, counters):
    c = np.ascontiguousarray(counters, dtype=np.uint64)
    _check(h, load().ravel_set_state(h, c.ctypes.data), "ravel_set_state")


def ravel_step_kernel_count(h) -> int:
    return int(load().ravel_step_kernel_count(h))


def ravel_status_string(status: int) -> str:
    return load().ravel_status_string(status).decode()


def ravel_last_error(h) -> str:
    return load().ravel_last_error(h).decode()


# ---- the 8-bit context cache (include/ravel_cache.h)


def current_stream_getter():
    """A function of a device's index that gives its current stream as an
    address.  (torch.cuda.current_stream makes an object first: 3 us of a call's
    13.)"""
    import torch
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return get if get is not None else lambda device: torch.cuda.current_stream(device).cuda_stream


def new_tensor(shape, dtype, device, stream, zeros=False):
    """A new tensor of the stream that is going to write it."""
    import torch
    make = torch.zeros if zeros else torch.empty
    if stream is None:
        return make(shape, dtype=dtype, device=device)
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    with torch.cuda.stream(stream):
        return make(shape, dtype=dtype, device=device)


def _check_cache(c, status: int, what: str):
    if status != 0:
        raise RavelError(status, f"{what}: {load().ravel_cache_last_error(c).decode()}")


class CacheArguments:
    """What the calls on a cache look over: types, shapes, strides and device of
    their tensors.  (The library takes addresses: what does not fit is read or
    written past its end.)"""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: int, device: int):
        import torch
        self.n_q_heads, self.n_kv_heads, self.head_dim = n_q_heads, n_kv_heads, head_dim
        self.dtype = torch.bfloat16 if dtype == RAVEL_BF16 else torch.float32
        self.int32, self.float32 = torch.int32, torch.float32
        self.device = torch.device("cuda", device)
        self.index = device

    def rows(self, x, heads: int, name: str):
        """Strides (robot, token) of a [batch, n, heads, head_dim] tensor whose heads are
        contiguous; 0 where there is one robot or one token, whose stride means nothing."""
        shape = x.shape
        if x.dtype is not self.dtype or len(shape) != 4 or shape[2] != heads or shape[3] != self.head_dim or \
                x.get_device() != self.index:
            raise ValueError(f"{name} must be [batch, n, {heads}, {self.head_dim}] of dtype {self.dtype} on {self.device}, "
                             f"got {tuple(shape)} of {x.dtype} on {x.device}")
        robot, token, head, dim = x.stride()
        if dim != 1 or (head != self.head_dim and heads > 1):
            raise ValueError(f"{name}: the heads of a token must be contiguous")
        return robot if shape[0] > 1 else 0, token if shape[1] > 1 else 0

    def ints(self, x, batch: int, name: str):
        """Address of an int32 tensor [batch], or None."""
        if x is None:
            return None
        if x.dtype is not self.int32 or x.shape != (batch,) or x.get_device() != self.index or not x.is_contiguous():
            raise ValueError(f"{name} must be a contiguous int32 tensor [{batch}] on {self.device}")
        return x.data_ptr()

    def mass(self, mass, batch):
        """Address and length of a mass's rows."""
        shape = mass.shape
        if len(shape) != 3 or (batch is not None and shape[0] != batch) or shape[1] != self.n_kv_heads or \
                mass.dtype is not self.float32 or mass.get_device() != self.index or not mass.is_contiguous():
            raise ValueError(f"mass must be a contiguous float32 tensor [{'batch' if batch is None else batch}, "
                             f"{self.n_kv_heads}, tokens] on {self.device}, got {tuple(shape)} of {mass.dtype}")
        return mass.data_ptr(), shape[2]

    def dense(self, x, shape: tuple, dtype, name: str):
        """Address of a contiguous tensor of that shape, or None."""
        if x is None:
            return None
        if x.dtype is not dtype or x.shape != shape or x.get_device() != self.index or not x.is_contiguous():
            raise ValueError(f"{name} must be a contiguous tensor {list(shape)} of dtype {dtype} on {self.device}, "
                             f"got {tuple(x.shape)} of {x.dtype} on {x.device}")
        return x.data_ptr()


def _arguments(c) -> CacheArguments:
    # (an attribute of the handle, not a class of its own, which ctypes takes 60 ns longer to pass)
    a = getattr(c, "arguments", None)
    if a is None:
        raise ValueError("not a handle that ravel_cache_create returned")
    return a


def ravel_cache_create(layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, max_tokens: int, max_batch: int,
                       max_queries: int, dtype: int = RAVEL_BF16, device: int = 0):
    c = RavelCacheConfig(layers, n_q_heads, n_kv_heads, head_dim, max_tokens, max_batch, max_queries, dtype)
    h = C.c_void_p()
    st = load().ravel_cache_create(C.byref(c), device, C.byref(h))
    if st != 0:
        raise RavelError(st, "ravel_cache_create failed (see stderr)")
    h.arguments = CacheArguments(n_q_heads, n_kv_heads, head_dim, dtype, device)
    return h


def ravel_cache_destroy(c):
    load().ravel_cache_destroy(c)


def ravel_cache_reset(c):
    _check_cache(c, load().ravel_cache_reset(c), "ravel_cache_reset")


def ravel_cache_append(c, layer: int, k, v, starts=None, counts=None, stream=None):
    """k, v [B, n, Hkv, hd] with the same strides; see ravel_cache.h."""
    a = _arguments(c)
    rs, ts = a.rows(k, a.n_kv_heads, "k")
    if v.shape != k.shape or a.rows(v, a.n_kv_heads, "v") != (rs, ts):
        raise ValueError("k and v must have the same shape and strides")
    B, n = k.shape[:2]
    _check_cache(c, load().ravel_cache_append(c, layer, B, n, k.data_ptr(), v.data_ptr(), rs, ts, a.ints(starts, B, "starts"),
                                              a.ints(counts, B, "counts"), _stream_ptr(stream)), "ravel_cache_append")


def ravel_cache_attend(c, layer: int, q, out, lengths, counts, max_length: int, causal: bool = True, window: int = 0,
                       sinks: int = 0, scale: float = 0.0, mass=None, add_mass: bool = False, stream=None):
    """q, out [B, n, Hq, hd]; mass float32 [B, Hkv, >= max_length] or None; see ravel_cache.h."""
    a = _arguments(c)
    qrs, qts = a.rows(q, a.n_q_heads, "q")
    ors, ots = a.rows(out, a.n_q_heads, "out")
    if out.shape != q.shape:
        raise ValueError("out must have q's shape")
    B, n = q.shape[:2]
    if lengths is None:
        raise ValueError("lengths must be a contiguous int32 CUDA tensor")
    mp, ms = a.mass(mass, B) if mass is not None else (None, 0)
    _check_cache(c, load().ravel_cache_attend(c, layer, B, n, q.data_ptr(), qrs, qts, out.data_ptr(), ors, ots,
                                              a.ints(lengths, B, "lengths"), a.ints(counts, B, "counts"), max_length,
                                              int(causal), window, sinks, scale, mp, ms, int(add_mass), _stream_ptr(stream)),
                 "ravel_cache_attend")


def ravel_cache_evict(c, layer: int, to, to_layer: int, lengths, mass, keep: int, sinks: int, recent: int, new_lengths,
                      index, new_mass=None, stream=None):
    """mass float32 [B, Hkv, tokens]; index int32 and new_mass float32 [B, Hkv, keep]; see ravel_cache.h."""
    a = _arguments(c)
    _arguments(to)
    mp, ms = a.mass(mass, None)
    B = mass.shape[0]
    kept = (B, a.n_kv_heads, keep)
    _check_cache(c, load().ravel_cache_evict(
        c, layer, to, to_layer, B, a.ints(lengths, B, "lengths"), mp, ms, keep, sinks, recent,
        a.ints(new_lengths, B, "new_lengths"), a.dense(index, kept, a.int32, "index"),
        a.dense(new_mass, kept, a.float32, "new_mass"), _stream_ptr(stream)), "ravel_cache_evict")


def ravel_cache_read(c, layer: int, k, v, firsts=None, lengths=None, stream=None):
    """k, v [B, Hkv, n, hd], contiguous, written; see ravel_cache.h."""
    a = _arguments(c)
    if len(k.shape) != 4:
        raise ValueError(f"k must be [batch, {a.n_kv_heads}, n, {a.head_dim}], got {tuple(k.shape)}")
    B, n = k.shape[0], k.shape[2]
    held = (B, a.n_kv_heads, n, a.head_dim)
    _check_cache(c, load().ravel_cache_read(c, layer, B, n, a.ints(firsts, B, "firsts"), a.ints(lengths, B, "lengths"),
                                            a.dense(k, held, a.dtype, "k"), a.dense(v, held, a.dtype, "v"),
                                            _stream_ptr(stream)), "ravel_cache_read")


_INT_MAX = (1 << 31) - 1


def _fit_ints(what: str, *values):
    """ctypes passes the low 32 bits of what does not fit into an int."""
    for x in values:
        if not -_INT_MAX <= x <= _INT_MAX:
            raise ValueError(f"{what}: {x} is beyond 2^31 - 1")


def ravel_cache_append_rotary(c, layer: int, rotary, q, q_out, k, v, starts=None, positions=None, counts=None, stream=None):
    """q, q_out [B, n, Hq, hd] (or None), k, v [B, n, Hkv, hd]; positions int32 [B, n]; see ravel_decode.h."""
    a = _arguments(c)
    if getattr(rotary, "rotary", None) is None:
        raise ValueError("not a handle that ravel_rotary_create returned")
    krs, kts = a.rows(k, a.n_kv_heads, "k")
    vrs, vts = a.rows(v, a.n_kv_heads, "v")
    shape = k.shape
    if v.shape != shape:
        raise ValueError("k and v must have the same shape")
    B, n = shape[0], shape[1]
    _fit_ints("ravel_cache_append_rotary", layer, B, n)
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    qp = qop = None
    qrs = qts = qors = qots = 0
    if q is not None:
        qrs, qts = a.rows(q, a.n_q_heads, "q")
        qors, qots = a.rows(q_out, a.n_q_heads, "q_out")
        if q.shape[:2] != shape[:2] or q_out.shape != q.shape:
            raise ValueError("q and q_out must have as many tokens as k")
        qp, qop = q.data_ptr(), q_out.data_ptr()
    _check_cache(c, load().ravel_cache_append_rotary(
        c, layer, rotary, B, n, qp, qrs, qts, qop, qors, qots, k.data_ptr(), krs, kts, v.data_ptr(), vrs, vts,
        a.ints(starts, B, "starts"), a.dense(positions, (B, n), a.int32, "positions"), a.ints(counts, B, "counts"),
        _stream_ptr(stream)), "ravel_cache_append_rotary")


# ---- rotary positions, 4-bit products, drawing tokens (include/ravel_decode.h)


def _check_decode(status: int, what: str):
    if status != 0:
        raise RavelError(status, f"{what}: {load().ravel_decode_last_error().decode()}")


class _Types:
    """torch's types, looked up once (an import statement takes 0.5 us of a call)."""
    bf16 = f32 = i32 = u8 = get_device = None

    @classmethod
    def look_up(cls):
        import torch
        cls.f32, cls.i32, cls.u8 = torch.float32, torch.int32, torch.uint8
        cls.get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        cls.bf16 = torch.bfloat16   # (the last: says that all are there)
        return cls


def _types():
    return _Types if _Types.bf16 is not None else _Types.look_up()


def _row_dtype(t, name: str) -> int:
    types = _types()
    if t.dtype is types.bf16:
        return RAVEL_BF16
    if t.dtype is types.f32:
        return RAVEL_FP32
    raise ValueError(f"{name} must be bfloat16 or float32, got {t.dtype}")


def _flat(t, shape: tuple, dtype, device: int, name: str):
    """Address of a contiguous CUDA tensor of that shape, or None."""
    if t is None:
        return None
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous():
            return t.data_ptr()
        got = f"{tuple(t.shape)} of {t.dtype} on {t.device}"
    except AttributeError:
        got = repr(t)
    raise ValueError(f"{name} must be a contiguous tensor {list(shape)} of {dtype} on cuda:{device}, got {got}")


def _matrix(t, rows: int, cols: int, device: int, name: str, wide: bool = False) -> int:
    """Row stride (an int; wide: a long long) of a [rows, cols] tensor whose rows are contiguous; of
    a single row, whose stride means nothing, the next multiple of 8."""
    stride = t.stride()
    if len(stride) != 2 or t.shape != (rows, cols) or t.get_device() != device or (stride[1] != 1 and cols > 1):
        raise ValueError(f"{name} must be [{rows}, {cols}] on cuda:{device} with contiguous rows, got {tuple(t.shape)} on {t.device}")
    if rows > _INT_MAX or cols > _INT_MAX or (stride[0] > _INT_MAX and rows > 1 and not wide):
        raise ValueError(f"{name}: more than 2^31 - 1 rows, columns, or values from one row to the next")
    if rows < 2:
        return -(-cols // 8) * 8
    if stride[0] < cols:
        raise ValueError(f"{name}: rows overlap")
    return stride[0]


def ravel_rotary_create(dims: int, base: float = 10000.0, interleaved: bool = False, factor: float = 1.0,
                        original_length: float = 0.0, low: float = 1.0, high: float = 32.0, amplitude: float = 1.0,
                        frequencies=None, device: int = 0):
    f = None
    _fit_ints("ravel_rotary_create", dims, device)
    if frequencies is not None:
        f = np.ascontiguousarray(frequencies, dtype=np.float64)
        if f.shape != (dims // 2,):
            raise ValueError(f"frequencies must be [{dims // 2}], got {f.shape}")
    c = RavelRotaryConfig(dims, int(interleaved), base, factor, original_length, low, high, amplitude,
                          None if f is None else f.ctypes.data_as(C.POINTER(C.c_double)))
    h = C.c_void_p()
    _check_decode(load().ravel_rotary_create(C.byref(c), device, C.byref(h)), "ravel_rotary_create")
    h.rotary = (dims, device)
    return h


def ravel_rotary_destroy(r):
    load().ravel_rotary_destroy(r)


def _heads(x, device: int, name: str):
    """Strides (robot, token) of a [batch, n, heads, hd] tensor whose heads are contiguous."""
    shape, stride = x.shape, x.stride()
    if len(shape) != 4 or x.get_device() != device:
        raise ValueError(f"{name} must be [batch, n, heads, head_dim] on cuda:{device}, got {tuple(shape)} on {x.device}")
    robot, token, head, dim = stride
    if (dim != 1 and shape[3] > 1) or (head != shape[3] and shape[2] > 1):
        raise ValueError(f"{name}: the heads of a token must be contiguous")
    if shape[0] > _INT_MAX or shape[1] > _INT_MAX or shape[2] > _INT_MAX or shape[3] > _INT_MAX:
        raise ValueError(f"{name}: sizes must be below 2^31")
    return robot if shape[0] > 1 else 0, token if shape[1] > 1 else 0


def ravel_rotary_apply(r, x, out, starts=None, positions=None, counts=None, stream=None):
    """x, out [B, n, heads, hd]; see ravel_decode.h."""
    if getattr(r, "rotary", None) is None:
        raise ValueError("not a handle that ravel_rotary_create returned")
    device = r.rotary[1]
    xr, xt = _heads(x, device, "x")
    if out is x:
        outr, outt = xr, xt
    else:
        outr, outt = _heads(out, device, "out")
        if out.shape != x.shape or out.dtype is not x.dtype:
            raise ValueError("out must have x's shape and dtype")
    B, n, heads, hd = x.shape
    i32 = _types().i32
    status = load().ravel_rotary_apply(
        r, B, n, heads, hd, _row_dtype(x, "x"), x.data_ptr(), xr, xt, out.data_ptr(), outr, outt,
        _flat(starts, (B,), i32, device, "starts"), _flat(positions, (B, n), i32, device, "positions"),
        _flat(counts, (B,), i32, device, "counts"), _stream_ptr(stream))
    if status:
        _check_decode(status, "ravel_rotary_apply")


def ravel_w4_create(N: int, K: int, group: int = 128, device: int = 0):
    h = C.c_void_p()
    _fit_ints("ravel_w4_create", N, K, group, device)
    _check_decode(load().ravel_w4_create(N, K, group, device, C.byref(h)), "ravel_w4_create")
    h.w4 = (N, K, group, device)
    return h


def ravel_w4_destroy(w):
    load().ravel_w4_destroy(w)


def ravel_w4_reset(w):
    _check_decode(load().ravel_w4_reset(w), "ravel_w4_reset")


def _w4(w):
    a = getattr(w, "w4", None)
    if a is None:
        raise ValueError("not a handle that ravel_w4_create returned")
    return a


def ravel_w4_load(w, codes, scales, zeros, stream=None):
    """codes uint8 [N, (K + 1) // 2], scales bfloat16 and zeros uint8 [N, groups]; see ravel_decode.h."""
    N, K, group, device = _w4(w)
    groups, types = -(-K // group), _types()
    _check_decode(load().ravel_w4_load(
        w, _flat(codes, (N, (K + 1) // 2), types.u8, device, "codes"), _flat(scales, (N, groups), types.bf16, device, "scales"),
        _flat(zeros, (N, groups), types.u8, device, "zeros"), _stream_ptr(stream)), "ravel_w4_load")


def ravel_w4_quantize(W, group: int, codes, scales, zeros, stream=None):
    """Nearest codes of W [N, K]; see ravel_decode.h."""
    import torch
    device = W.get_device()
    if W.dim() != 2 or device < 0:
        raise ValueError(f"W must be a CUDA tensor [N, K], got {tuple(W.shape)} on {W.device}")
    N, K = W.shape
    _fit_ints("ravel_w4_quantize", group)
    ldw = _matrix(W, N, K, device, "W")
    groups = -(-K // group)
    with torch.cuda.device(device):
        _check_decode(load().ravel_w4_quantize(
            W.data_ptr(), N, K, ldw, _row_dtype(W, "W"), group, _flat(codes, (N, (K + 1) // 2), torch.uint8, device, "codes"),
            _flat(scales, (N, groups), torch.bfloat16, device, "scales"), _flat(zeros, (N, groups), torch.uint8, device, "zeros"),
            _stream_ptr(stream)), "ravel_w4_quantize")


def ravel_w4_read(w, out, stream=None):
    """out [N, K], written; see ravel_decode.h."""
    N, K, _, device = _w4(w)
    ldo = _matrix(out, N, K, device, "out")
    _check_decode(load().ravel_w4_read(w, out.data_ptr(), ldo, _row_dtype(out, "out"), _stream_ptr(stream)), "ravel_w4_read")


W4_EPILOGUES = {"store": 0, "silu": 1, "add": 2, "geglu": 3}


def ravel_w4_gemm(w, X, epi: int, out, bias=None, stream=None):
    """out (op)= X [M, K] times the matrix's rows (+ bias); see ravel_decode.h."""
    N, K, _, device = _w4(w)
    types = _types()
    if X.dtype is not types.bf16:
        raise ValueError(f"X must be bfloat16, got {X.dtype}")
    if not 0 <= epi <= 3:
        raise ValueError(f"unknown epilogue {epi}")
    M = X.shape[0]
    lda = _matrix(X, M, K, device, "X")
    ldo = _matrix(out, M, N // 2 if epi == 3 else N, device, "out")
    status = load().ravel_w4_gemm(w, X.data_ptr(), M, lda, epi, out.data_ptr(), ldo, _row_dtype(out, "out"),
                                       _flat(bias, (N,), types.f32, device, "bias"), _stream_ptr(stream))
    if status:
        _check_decode(status, "ravel_w4_gemm")


def ravel_draw_tokens(logits, u, temperature, top_k, top_p, min_p, tokens, log_probs=None, stream=None):
    """logits [B, V]; the others [B] or None; tokens int32 and log_probs float32 [B], written; see ravel_decode.h."""
    types = _types()
    device = logits.get_device()
    if logits.dim() != 2 or device < 0:
        raise ValueError(f"logits must be a CUDA tensor [batch, vocab], got {tuple(logits.shape)} on {logits.device}")
    B, V = logits.shape
    row = _matrix(logits, B, V, device, "logits", wide=True)
    f32, i32, one = types.f32, types.i32, (B,)
    if u is None or tokens is None:
        raise ValueError("u and tokens must be given")
    args = (logits.data_ptr(), B, V, row, _row_dtype(logits, "logits"), _flat(u, one, f32, device, "u"),
            _flat(temperature, one, f32, device, "temperature"), _flat(top_k, one, i32, device, "top_k"),
            _flat(top_p, one, f32, device, "top_p"), _flat(min_p, one, f32, device, "min_p"), _flat(tokens, one, i32, device, "tokens"),
            _flat(log_probs, one, f32, device, "log_probs"), _stream_ptr(stream))
    if types.get_device() == device:
        status = load().ravel_draw_tokens(*args)
    else:
        import torch
        with torch.cuda.device(device):
            status = load().ravel_draw_tokens(*args)
    if status:
        _check_decode(status, "ravel_draw_tokens")
