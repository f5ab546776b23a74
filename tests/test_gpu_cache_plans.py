"""The 8-bit context cache's attention where launches are planned otherwise: many
splits (joined in shared memory or through L2), caches with room to spare, long
ones, addresses past 32 bits, references that grow from tile to tile.  Against the
fp64 reference, within the tolerances of test_gpu_cache.py."""
import numpy as np
import pytest

from oracle import cache as ref
from tests.test_gpu_cache import Pair, _ints, _lib, _np, _rand, _within, check  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _growing(layout, batch, n, tokens, step, order, seed=0):
    """Keys whose scores rise (or fall) by about `step` in the log2 domain from one tile of 128 tokens
    to the next, values of which one block in three is 2^10 or 2^20 above the others; robots alike."""
    hq, hkv, hd = layout
    rng = np.random.default_rng(seed)
    u = rng.choice([-1.0, 1.0], (hkv, hd)) / np.sqrt(hd)
    tile = np.arange(tokens) // 128
    tile = {"up": tile, "down": tile.max() - tile, "mixed": rng.permutation(tile.max() + 1)[tile]}[order]
    # score of q = s u against k = a u: s a / sqrt(hd)
    k = (tile * step * np.log(2))[:, None, None] * u + 0.3 * rng.standard_normal((tokens, hkv, hd))
    q = np.sqrt(hd) * np.repeat(u, hq // hkv, 0) * rng.choice([1.0, 1.0, 0.4, -1.0], (n, hq, 1)) + 0.3 * rng.standard_normal((n, hq, hd))
    v = rng.standard_normal((tokens, hkv, hd)) * 2.0 ** (10 * (np.arange(tokens) // 16 % 7 % 3))[:, None, None]
    return [torch.from_numpy(x).to(torch.bfloat16).cuda()[None].expand(batch, *x.shape).contiguous() for x in (q, k, v)]


@pytest.mark.parametrize("layout,n,batch,tokens", [((4, 1, 40), 330, 8, 700), ((16, 4, 64), 300, 3, 700), ((8, 1, 64), 300, 2, 3000),
                                                   ((4, 2, 128), 300, 9, 700), ((3, 1, 192), 300, 11, 700), ((8, 1, 256), 300, 17, 700)])
@pytest.mark.parametrize("step,order", [(12, "up"), (40, "up"), (15, "mixed"), (25, "down")])
def test_references_that_grow_from_tile_to_tile(layout, n, batch, tokens, step, order):
    """Six tiles to an item, or splits of several; with 17 robots several items to a CTA."""
    p = Pair(layout, "bf16", tokens, batch, queries=n)
    q, k, v = _growing(layout, batch, n, tokens, step, order)
    p.cache.append(0, k, v)
    one = Pair(layout, "bf16", 16, 1)
    one.lengths, one.held = [tokens], ref.Held(1, layout[1], tokens, layout[2])
    one.held.append(_np(k[:1]), _np(v[:1]), [0], [tokens])
    L = _ints([tokens] * batch)
    for causal, window, sinks in ((False, 0, 0), (True, 500, 3)):
        mass = torch.zeros((batch, layout[1], tokens), device="cuda")
        out = p.cache.attend(0, q, L, causal=causal, window=window, sinks=sinks, mass=mass)
        for b in range(1, batch):
            assert torch.equal(out[b], out[0]) and torch.equal(mass[b], mass[0])
        _within(one, out[:1], q[:1], n, causal, window, sinks, mass[:1])


@pytest.mark.parametrize("layout,n", [((6, 2, 40), 33), ((16, 4, 64), 21), ((8, 1, 64), 60), ((8, 2, 128), 40), ((5, 1, 192), 26),
                                      ((8, 1, 256), 50), ((8, 1, 256), 3)])
def test_many_rows_in_more_splits_than_a_cluster_holds(layout, n):
    tokens = 4700
    p = Pair(layout, "bf16", 5000, 2, queries=n, lengths=[tokens, 1203], seed=31, scale=1.5)
    q = _rand((2, n, layout[0], layout[2]), 32, "bf16", 2.0)
    L, counts = _ints(p.lengths), [n, n - 2]
    first = {}
    for turn in range(2):        # plans in turn on one cache: nothing is left behind by one for the next
        for causal, window, sinks, most in ((False, 0, 0, None), (True, 0, 0, None), (True, 1500, 5, None), (True, 0, 0, 4700),
                                            (True, 300, 140, None)):
            mass = torch.full((2, layout[1], 5000), -1.0, device="cuda")
            out = p.cache.attend(0, q, L, counts=_ints(counts), causal=causal, window=window, sinks=sinks, mass=mass, max_length=most)
            key = (causal, window, sinks, most)
            if turn == 0:
                first[key] = out.clone(), mass.clone()
                _within(p, out, q, n, causal, window, sinks, mass[:, :, :most or 5000], counts)
            assert torch.equal(out, first[key][0]) and torch.equal(mass, first[key][1])
        # one robot alone (more splits still), and a short bound (few)
        out = p.cache.attend(0, q[:1], L[:1])
        _within_first(p, out, q, n)
        if n >= 20:
            p2 = p.cache.attend(0, q[1:], _ints([n]), max_length=128)
            assert torch.isfinite(p2).all()


def _within_first(pair, got, q, n):
    one = Pair.__new__(Pair)
    one.layout, one.dtype, one.batch, one.lengths = pair.layout, pair.dtype, 1, pair.lengths[:1]
    one.held = ref.Held(1, pair.layout[1], 16, pair.layout[2])
    one.held.k, one.held.v = pair.held.k[:1], pair.held.v[:1]
    _within(one, got, q[:1], n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout,n", [((8, 1, 256), 1), ((8, 1, 256), 2), ((5, 1, 192), 3), ((4, 2, 128), 1), ((16, 1, 128), 1),
                                      ((12, 1, 72), 1), ((16, 4, 64), 4)])
def test_few_rows_in_more_splits_than_a_cluster_holds(layout, n, dtype):
    p = Pair(layout, dtype, 6100, 2, queries=n, lengths=[6001, 2999], seed=51, scale=1.5)
    for causal, window, sinks in ((True, 0, 0), (False, 0, 0), (True, 4000, 7)):
        out, m = check(p, n, causal=causal, window=window, sinks=sinks, mass=True)
        again, m2 = check(p, n, causal=causal, window=window, sinks=sinks, mass=True)
        assert torch.equal(out, again) and torch.equal(m, m2)
    check(p, n, counts=[n, 0], mass=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [1, 3, 40])
@pytest.mark.parametrize("room", [816, 8192, 32768])
def test_a_robot_in_a_cache_with_room_to_spare(room, n, dtype):
    p = Pair((8, 1, 256), dtype, room, 1, queries=n, lengths=[816], seed=61)
    for more in (dict(), dict(causal=False), dict(window=200, sinks=4)):
        check(p, n, mass=True, **more)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout,n", [((4, 1, 64), 1), ((8, 1, 256), 2), ((4, 1, 64), 30)])
def test_positions_far_into_a_long_cache(layout, n, dtype):
    tokens = 130003
    p = Pair(layout, dtype, 131072, 1, queries=n, lengths=[tokens], seed=71)
    check(p, n, mass=True, q_scale=1.0)
    check(p, n, mass=True, window=70000, sinks=20, q_scale=3.0)


@pytest.mark.parametrize("dtype,n", [("bf16", 1), ("bf16", 40), ("fp32", 3)])
def test_rows_whose_addresses_pass_32_bits(dtype, n):
    """35 robots of 4 heads, 131072 tokens of room and 256 bytes a row: 4.7 GB of keys; the last robot's
    lie past 4 GB."""
    from paper_2609_34170_gb300 import ContextCache
    batch, hq, hkv, hd, tokens = 35, 4, 4, 256, 300
    cache = ContextCache(1, hq, hkv, hd, 131072, batch, n, dtype)
    small = Pair((hq, hkv, hd), dtype, 131072 // 128, 1, queries=n)
    k, v = _rand((1, tokens, hkv, hd), 1, dtype), _rand((1, tokens, hkv, hd), 2, dtype)
    q = _rand((1, n, hq, hd), 3, dtype, 2.0)
    counts = [0] * (batch - 1) + [tokens]
    at = [0] * (batch - 1) + [131072 - tokens - 5]      # (what lies before it is zeros)
    wide = [x.expand(batch, *x.shape[1:]) for x in (k, v)]
    cache.append(0, *wide, counts=_ints(counts))
    small.cache.append(0, k, v)
    small.held.append(_np(k), _np(v), [0], [tokens])
    small.lengths = [tokens]
    mass = torch.zeros((batch, hkv, 512), device="cuda")
    nothing = [0] * (batch - 1)
    out = cache.attend(0, q.expand(batch, *q.shape[1:]), _ints(counts), counts=_ints(nothing + [n]), max_length=512, mass=mass)
    check(small, n, q=q, mass=True)
    assert (out[:-1] == 0).all() and (mass[:-1] == 0).all()
    o, ms, W, size = ref.attend(_np(q), small.held, [tokens], [n])
    d = 2.0 ** -18 * size[..., None]
    lost = (2.0 ** -8, 2.0 ** -10) if dtype == "bf16" else (2.0 ** -22, 2.0 ** -20 + (tokens / 16 + 4) * 2.0 ** -22)
    assert (np.abs(_np(out)[-1:] - o) <= lost[0] * np.abs(o) + (lost[1] + 2 * d) * W).all()
    for got, held in zip(cache.read(0, batch, tokens, lengths=_ints(counts)), (small.held.k, small.held.v)):
        assert (got[:-1] == 0).all()
        np.testing.assert_array_equal(_np(got)[-1], held[0, :, :tokens])
    to = ContextCache(1, hq, hkv, hd, 131072, batch, n, dtype)
    kept, index, _ = cache.evict(0, to, 0, _ints(counts), mass, 100, 3, 5)
    _, want_index, _, held = ref.evict(small.held, [tokens], _np(mass)[-1:].astype(np.float32), 100, 3, 5)
    np.testing.assert_array_equal(index[-1:].cpu().numpy(), want_index)
    np.testing.assert_array_equal(_np(to.read(0, batch, 100, lengths=kept)[0])[-1], held.k[0, :, :100])
    cache.append(0, *wide, _ints(at), _ints(counts))
    got = cache.read(0, batch, tokens, firsts=_ints(at))[0]
    first = (at[-1] // 16 + 1) * 16 - at[-1]            # (its first block holds zeros as well)
    other = ref.Held(1, hkv, tokens + 32, hd)
    other.append(_np(k), _np(v), [at[-1] % 16], [tokens])
    np.testing.assert_array_equal(_np(got)[-1, :, first:], other.k[0, :, at[-1] % 16 + first:at[-1] % 16 + tokens])
