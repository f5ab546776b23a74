"""64-bit references of rotary positions, 4-bit products and drawing tokens,
written from their definitions (include/ravel_decode.h), numpy only."""
import math

import numpy as np


def frequencies(dims, base=10000.0, factor=1.0, original_length=0.0, low=1.0, high=32.0):
    out = []
    for i in range(dims // 2):
        f = base ** (-2.0 * i / dims)
        t = original_length * f / (2 * math.pi)
        if original_length and t >= high:
            out.append(f)
        elif original_length and t > low:
            g = (t - low) / (high - low)
            out.append(g * f + (1 - g) * f / factor)
        else:
            out.append(f / factor)
    return np.array(out)


def pairs(dims, interleaved):
    """Indices of the first and of the second dims of the pairs."""
    i = np.arange(dims // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + dims // 2)


def turn(x, positions, f, interleaved=False, amplitude=1.0):
    """x [B, n, H, hd] at positions [B, n]."""
    y = np.array(x, np.float64)
    first, second = pairs(2 * len(f), interleaved)
    a = np.asarray(positions, np.float64)[:, :, None, None] * f
    c, s = amplitude * np.cos(a), amplitude * np.sin(a)
    p, q = y[..., first].copy(), y[..., second].copy()
    y[..., first], y[..., second] = p * c - q * s, p * s + q * c
    return y


def pair_size(x, dims, interleaved):
    """|first| + |second| of each dim's pair (zero of dims that stay): what its error is relative to."""
    y = np.abs(np.array(x, np.float64))
    first, second = pairs(dims, interleaved)
    size = np.zeros_like(y)
    size[..., first] = size[..., second] = y[..., first] + y[..., second]
    return size


# ---- 4-bit weights


def bf16(x):
    """fp32 values rounded to bf16 (nearest, ties to even)."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000
    return u.astype(np.uint32).view(np.float32)


def unpack(codes, k):
    return np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)[:, :k]


def weights(codes, scales, zeros, k, group):
    """[N, K] in 64 bits of codes [N, (K + 1) // 2], scales and zeros [N, groups]."""
    at = np.arange(k) // group
    return (unpack(codes, k).astype(np.float64) - zeros[:, at]) * np.asarray(scales, np.float64)[:, at]


def quantize(w, group):
    """Codes [N, K], scales, zeros of a matrix, step by step in fp32 as defined."""
    w = np.asarray(w, np.float32)
    n, k = w.shape
    groups = -(-k // group)
    codes, scales, zeros = np.zeros((n, k), np.uint8), np.zeros((n, groups), np.float32), np.zeros((n, groups), np.uint8)
    for g in range(groups):
        part = w[:, g * group:(g + 1) * group]
        lo, hi = np.minimum(part.min(1), np.float32(0)), np.maximum(part.max(1), np.float32(0))
        s = bf16((hi - lo) / np.float32(15))
        some = s > 0
        safe = np.where(some, s, np.float32(1))
        z = np.where(some, np.clip(np.rint(-lo / safe), 0, 15), 0).astype(np.float32)
        c = np.clip(np.rint(part / safe[:, None] + z[:, None]), 0, 15)
        codes[:, g * group:(g + 1) * group] = np.where(some[:, None], c, 0)
        scales[:, g], zeros[:, g] = s, z
    return codes, scales, zeros


def pack(codes):
    if codes.shape[1] % 2:
        codes = np.concatenate([codes, np.zeros((codes.shape[0], 1), np.uint8)], 1)
    return codes[:, 0::2] | codes[:, 1::2] << 4


def gelu(g):
    return 0.5 * g * (1 + np.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def geglu_rows(y):
    """Gate and up columns of y [M, N]: blocks of 64 and 64."""
    blocks = y.reshape(y.shape[0], -1, 2, 64)
    return blocks[:, :, 0].reshape(y.shape[0], -1), blocks[:, :, 1].reshape(y.shape[0], -1)


# ---- drawing a token


def draw(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log-probability) of one row of logits."""
    x = np.asarray(x, np.float64)
    u, t, p, q = (float(v) for v in (u, temperature, top_p, min_p))
    if np.isnan(x).any() or (x == np.inf).any() or not np.isfinite(x).any() or not 0 <= u < 1 or not t < math.inf or \
            math.isnan(p) or math.isnan(q):
        return -1, -math.inf
    order = np.argsort(-x, kind="stable")
    if t < 2.0 ** -20:
        return int(order[0]), 0.0
    if top_k > 0:
        order = order[:top_k]
    top = x[order[0]]
    with np.errstate(over="ignore"):
        z = (x[order] - top) / t
    w = np.exp(z)
    if p < 1:
        total, run, stop = math.fsum(w), 0.0, len(w)
        cum = np.cumsum(w)
        reached = np.nonzero(cum >= max(p, 0.0) * total)[0]
        stop = int(reached[0]) + 1 if len(reached) else len(w)
        order, w, z = order[:stop], w[:stop], z[:stop]
    stays = w >= min(q, 1.0) if q > 0 else np.ones(len(w), bool)
    order, w, z = order[stays], w[stays], z[stays]
    by_index = np.argsort(order)
    cum = np.cumsum(w[by_index])
    at = int(np.nonzero(cum > u * cum[-1])[0][0])
    return int(order[by_index[at]]), float(z[by_index[at]] - math.log(cum[-1]))
