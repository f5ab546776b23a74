"""fp64 reference of the 8-bit context cache: what a block holds, attention over
held values, attention mass, eviction.  numpy only, from the definitions in
include/ravel_cache.h."""
from __future__ import annotations

import numpy as np

BLOCK, TOP, E_MIN = 16, 448.0, -100


def exponent(top: float) -> int:
    """The smallest e >= -100 with top <= 448 * 2^e."""
    e = E_MIN
    if top > 0:
        e = max(E_MIN, int(np.frexp(top / TOP)[1]) - 2)
        while top > TOP * 2.0 ** e:
            e += 1
    return e


def e4m3(x: np.ndarray) -> np.ndarray:
    """Round to 4 exponent and 3 mantissa bits (bias 7, subnormals), ties to even."""
    x = np.asarray(x, np.float64)
    _, ex = np.frexp(x)                       # |x| = m 2^ex, m in [0.5, 1)
    grid = 2.0 ** (np.maximum(ex - 1, -6) - 3)
    return np.round(x / grid) * grid


class Held:
    """One layer: keys and values [B, H, T, hd] as held, exponents [B, H, T / 16]."""

    def __init__(self, B, H, T, hd):
        T = -(-T // BLOCK) * BLOCK
        self.k, self.v = np.zeros((B, H, T, hd)), np.zeros((B, H, T, hd))
        self.ke, self.ve = np.zeros((B, H, T // BLOCK), int), np.zeros((B, H, T // BLOCK), int)

    def _block(self, b, h, blk, new_k, new_v, fresh):
        """Tokens `fresh` (bool [16]) of a block take new rows; those before the first of them stay."""
        s = slice(blk * BLOCK, (blk + 1) * BLOCK)
        first = int(np.argmax(fresh))
        bad = fresh & ~(np.isfinite(new_k).all(-1) & np.isfinite(new_v).all(-1))
        good = fresh & ~bad
        for x, rows, e, fill in ((self.k, new_k, self.ke, np.nan), (self.v, new_v, self.ve, 0.0)):
            n = exponent(np.abs(rows[good]).max() if good.any() else 0.0)
            if first:
                n = max(n, e[b, h, blk])
            held = x[b, h, s]
            held[:first] = e4m3(held[:first] * 2.0 ** -n) * 2.0 ** n
            held[good] = e4m3(rows[good] * 2.0 ** -n) * 2.0 ** n
            held[bad] = fill
            e[b, h, blk] = n

    def append(self, k, v, starts, counts):
        """k, v [B, n, H, hd]"""
        B, _, H, hd = k.shape
        for b in range(B):
            at, end = int(starts[b]), int(starts[b]) + int(counts[b])
            for blk in range(at // BLOCK, -(-end // BLOCK) if end > at else 0):
                pos = np.arange(blk * BLOCK, (blk + 1) * BLOCK)
                fresh = (pos >= at) & (pos < end)
                src = np.clip(pos - at, 0, k.shape[1] - 1)
                for h in range(H):
                    self._block(b, h, blk, k[b, src, h], v[b, src, h], fresh)


def visible(length, count, i, causal, window, sinks):
    """Positions that query i of `count` sees."""
    j = np.arange(length)
    if i >= count:
        return np.zeros(length, bool)
    if not causal:
        return np.ones(length, bool)
    p = length - count + i
    see = j <= p
    if window:
        see &= (j > p - window) | (j < sinks)
    return see


def attend(q, held: Held, lengths, counts, causal=True, window=0, sinks=0, scale=None):
    """q [B, n, Hq, hd] -> out, mass [B, H, T], and for error bounds: the
    weighted mean of |v| per output and the largest scale * sum |q k| per row."""
    B, n, Hq, hd = q.shape
    H, T = held.k.shape[1:3]
    G = Hq // H
    scale = 1.0 / np.sqrt(hd) if scale is None else scale
    out, spread = np.zeros((B, n, Hq, hd)), np.zeros((B, n, Hq, hd))
    size, mass = np.zeros((B, n, Hq)), np.zeros((B, H, T))
    for b in range(B):
        L = int(lengths[b])
        for i in range(min(n, int(counts[b]))):
            see = visible(L, int(counts[b]), i, causal, window, sinks)
            if not see.any():
                continue
            for h in range(Hq):
                k, v = held.k[b, h // G, :L][see], held.v[b, h // G, :L][see]
                s = scale * (k @ q[b, i, h])
                w = np.exp(s - s.max()) if np.isfinite(s).all() else np.full(len(s), np.nan)
                w = w / w.sum()
                out[b, i, h], spread[b, i, h] = w @ v, w @ np.abs(v)
                size[b, i, h] = scale * (np.abs(k) @ np.abs(q[b, i, h])).max()
                mass[b, h // G, np.flatnonzero(see)] += w
    return out, mass, spread, size


def evict(held: Held, lengths, mass, keep, sinks, recent):
    """-> new lengths [B], index [B, H, keep], mass [B, H, keep], the new Held"""
    B, H, _, hd = held.k.shape
    index, kept = np.full((B, H, keep), -1), np.zeros((B, H, keep))
    new = Held(B, H, keep, hd)
    rows = {n: np.zeros((B, keep, H, hd)) for n in "kv"}
    for b in range(B):
        L = int(lengths[b])
        for h in range(H):
            pick = np.arange(L)
            if L > keep:
                mid = np.arange(sinks, L - recent)
                m = mass[b, h, mid] + 0.0
                heavy = mid[np.lexsort((mid, -np.where(np.isnan(m), 0.0, m), ~np.isnan(m)))][:keep - sinks - recent]
                pick = np.sort(np.concatenate([np.arange(sinks), heavy, np.arange(L - recent, L)])).astype(int)
            index[b, h, :len(pick)] = pick
            kept[b, h, :len(pick)] = mass[b, h, pick]
            rows["k"][b, :len(pick), h], rows["v"][b, :len(pick), h] = held.k[b, h, pick], held.v[b, h, pick]
    new_lengths = np.minimum(np.asarray(lengths), keep)
    new.append(rows["k"], rows["v"], np.zeros(B, int), new_lengths)
    return new_lengths, index, kept, new
