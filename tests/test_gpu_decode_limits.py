"""Rotary positions, 4-bit products and drawing tokens at the ends of what their headers allow."""
import math

import numpy as np
import pytest

from tests.test_gpu_decode import _draws, _ints, _lib, _rand  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dims,interleaved", [(8, False), (4, True)])
def test_append_rotary_of_more_heads_than_half_a_grid(dims, interleaved):
    """As apply and append with fp32 between them; keys and queries of one launch would be 2 x 40000 rows of CTAs."""
    from paper_2609_34170_gb300 import ContextCache, Rotary
    heads, hd = 40000, 8
    r = Rotary(dims, interleaved=interleaved)
    cache, plain = (ContextCache(1, heads, heads, hd, 16, 1, 1, dtype) for dtype in ("bf16", "fp32"))
    q, k, v = (_rand((1, 3, heads, hd), s, "bf16") for s in (1, 2, 3))
    starts = _ints([5])
    got = cache.append_rotary(0, r, q, k, v, starts)
    plain.append(0, r.apply(k.float(), starts=starts), v.float(), starts)
    assert torch.equal(got, r.apply(q, starts=starts))
    for a, b in zip(cache.read(0, 1, 8), plain.read(0, 1, 8)):
        assert torch.equal(a.float(), b)


def test_append_rotary_refuses_queries_beyond_what_it_counts():
    """Places in a token's queries are counted in 32 bits.  (The addresses are never looked at.)"""
    from paper_2609_34170_gb300 import ContextCache, Rotary, load
    heads, hd = 1 << 23, 256
    cache, r = ContextCache(1, heads, 1, hd, 16, 1), Rotary(hd)
    k = _rand((1, 1, 1, hd), 0, "bf16")
    assert load().ravel_cache_append_rotary(cache.handle, 0, r.handle, 1, 1, 1 << 20, 0, 0, 1 << 20, 0, 0, k.data_ptr(), 0, 0, k.data_ptr(), 0,
                                            0, None, None, None, 0) == 2
    assert cache.append_rotary(0, r, None, k, k) is None   # keys alone are not limited
    held = cache.read(0, 1, 1)[0]
    other = ContextCache(1, 1, 1, hd, 16, 1)
    other.append_rotary(0, r, None, k, k)
    assert torch.equal(held, other.read(0, 1, 1)[0])


@pytest.mark.parametrize("low,high", [(2.0 ** -20, 1.0), (1.0, 2.0 ** 64), (2.0 ** 64, 2.0 ** 110), (2.0 ** 110, 3.4e38)])
def test_weights_at_every_temperature(low, high):
    """Two tokens, and u the float next to the share of the first: which one is drawn says on which side of u the share
    lies.  Weights are good to 2^-42 (1e-12 from there on is decided), u and shares to 2^-25."""
    rng = np.random.default_rng(1)
    t = np.exp(rng.uniform(math.log(low), math.log(high), 4000)).astype(np.float32)
    first = (rng.uniform(0.0, 1.0, 4000) * np.minimum(8.0 * t.astype(np.float64), 3.4e38)).astype(np.float32)
    second = np.maximum(first.astype(np.float64) - rng.uniform(0.2, 3.0, 4000) * t, -3.4e38).astype(np.float32)
    share = 1 / (1 + np.exp((second.astype(np.float64) - first) / t))
    u = share.astype(np.float32)
    clear = (np.abs(u - share) > 1e-12) & (u < 1)
    assert clear.sum() > 3900
    _draws(torch.from_numpy(np.stack([first, second], 1)[clear]).cuda(), u[clear], t=t[clear])


def test_min_p_at_temperatures_whose_border_is_far_below_the_row():
    """T ln(min_p) is beyond fp32, the border that it makes is not: 3.4e38 - 4e38 lies within the row."""
    rng = np.random.default_rng(0)
    x = torch.from_numpy(rng.uniform(-3.39e38, 3.39e38, (8, 5000)).astype(np.float32)).cuda()
    x[:, 7] = 3.4e38
    t = [1e38, 1e38, 2e38, 2e38, 3.3e38, 3.3e38, 1.5e38, 1e20]
    q = [math.exp(-4), 0.03, 0.15, 0.2, 0.17, 0.3, 0.07, 0.5]
    for u in (0.0, 0.3, 0.7, 1 - 2.0 ** -24):
        _draws(x, [u] * 8, t=t, q=q)
        _draws(x, [u] * 8, t=t, q=q, p=[0.9] * 8)
        _draws(x, [u] * 8, t=t, q=q, k=[400] * 8)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout,dims,interleaved", [((8, 1, 256), 256, False), ((16, 4, 64), 64, True), ((6, 2, 40), 16, True),
                                                     ((4, 4, 128), 34, False), ((20, 1, 64), 64, False)])
@pytest.mark.parametrize("n", [1, 5, 16, 17, 40])
def test_append_rotary_in_place_leaves_the_rest_of_the_projection(layout, dims, interleaved, dtype, n):
    """Queries turned in place, columns of one projection: its keys and values stay as they were, and so do query rows from
    counts[b] on and those of a robot that is left out."""
    from paper_2609_34170_gb300 import ContextCache, Rotary
    hq, hkv, hd = layout
    r = Rotary(dims, interleaved=interleaved)
    cache = ContextCache(1, hq, hkv, hd, 64, 4, 1, dtype)
    qkv = _rand((4, n, hq + 2 * hkv, hd), n, dtype, 2.0)
    was = qkv.clone()
    counts = [n, n // 2, 0, n]
    starts = [3, 20, 9, 65 - n]   # (the last robot's tokens would pass the cache's end)
    q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
    assert cache.append_rotary(0, r, q, k, v, _ints(starts), counts=_ints(counts), q_out=q) is q
    torch.cuda.synchronize()
    cache.reset()
    turned = r.apply(was[:, :, :hq], starts=_ints(starts))
    for b in range(4):
        c = counts[b] if b < 3 else 0
        assert torch.equal(q[b, :c], turned[b, :c]) and torch.equal(q[b, c:], was[b, c:, :hq])
    assert torch.equal(qkv[:, :, hq:], was[:, :, hq:])
