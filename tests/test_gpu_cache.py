"""The 8-bit context cache on the GPU against the fp64 reference.

Stored values, eviction's choice and read-back are equal bit for bit.  Attention
is compared per element within

  bf16: 2^-8 |o| + (2^-10 + 2 d) W        fp32: 2^-22 |o| + (2^-20 + (T / 16 + 4) 2^-22 + 2 d) W

where W is the softmax-weighted mean of |v| of that output, d the error of a
score (2^-18 of the row's largest scale * sum |q k|: 23-bit operands, up to 64
truncating fp32 sums per score), 2^-8 |o| the output's rounding (half a unit,
2^-9, doubled), 2^-10 / 2^-20 twice the rounding of P (11 bits, or 22 in two pieces), and
(T / 16 + 4) 2^-22 the truncating sums of P V, one per 16 tokens and some to join
them.  Mass: (2^-18 + 2 d) of its own value plus rounding of the sum."""
import numpy as np
import pytest

from oracle import cache as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LAYOUTS = [(8, 1, 256), (16, 4, 64), (6, 2, 40), (4, 4, 128), (3, 1, 72), (5, 1, 192), (20, 1, 64), (1, 1, 8)]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_34170_gb300 import build, load
    build.build()
    load()


def _dt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _rand(shape, seed, dtype, scale=1.0):
    x = torch.from_numpy(np.random.default_rng(seed).standard_normal(shape) * scale)
    return x.to(_dt(dtype)).cuda()


def _ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def _np(t):
    return t.detach().double().cpu().numpy()


class Pair:
    """A cache and its reference, filled with the same tokens."""

    def __init__(self, layout, dtype, tokens, batch, queries=1, lengths=None, seed=0, scale=1.0, layers=1, pad=float("nan")):
        from paper_2609_34170_gb300 import ContextCache
        hq, hkv, hd = layout
        self.layout, self.dtype, self.batch = layout, dtype, batch
        self.cache = ContextCache(layers, hq, hkv, hd, tokens, batch, queries, dtype)
        self.held = ref.Held(batch, hkv, tokens, hd)
        if lengths is not None:
            self.lengths = list(lengths)
            n = max(self.lengths)
            if n:
                k, v = _rand((batch, n, hkv, hd), seed, dtype, scale), _rand((batch, n, hkv, hd), seed + 1, dtype)
                for b, m in enumerate(self.lengths):
                    k[b, m:] = pad
                    v[b, m:] = pad
                self.cache.append(layers - 1, k, v, counts=_ints(self.lengths))
                self.held.append(_np(k), _np(v), [0] * batch, self.lengths)


def check(pair, n, counts=None, causal=True, window=0, sinks=0, mass=False, seed=7, q=None, layer=0, q_scale=2.0, **more):
    hq, hkv, hd = pair.layout
    q = _rand((pair.batch, n, hq, hd), seed, pair.dtype, q_scale) if q is None else q
    cnt = [n] * pair.batch if counts is None else list(counts)
    m = torch.full((pair.batch, hkv, pair.cache.max_tokens), -7.0, device="cuda") if mass else None
    out = pair.cache.attend(layer, q, _ints(pair.lengths), counts=None if counts is None else _ints(cnt), causal=causal,
                            window=window, sinks=sinks, mass=m, **more)
    torch.cuda.synchronize()
    o, ms, W, size = ref.attend(_np(q), pair.held, pair.lengths, cnt, causal, window, sinks)
    d = 2.0 ** -18 * size[..., None]
    T = max(pair.lengths + [1])
    if pair.dtype == "bf16":
        tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -10 + 2 * d) * W
    else:
        tol = 2.0 ** -22 * np.abs(o) + (2.0 ** -20 + (T / 16 + 4) * 2.0 ** -22 + 2 * d) * W
    got = _np(out)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(o))
    err = np.abs(got - o) - tol
    assert not np.nanmax(err) > 1e-37, (np.nanmax(np.abs(got - o)), np.nanmax(tol), np.unravel_index(np.nanargmax(err), err.shape))
    if mass:
        gm = _np(m)[:, :, :ms.shape[2]]
        want = np.zeros_like(gm)
        want[:, :, :] = ms[:, :, :gm.shape[2]]
        dm = 2 * 2.0 ** -18 * np.nanmax(np.concatenate([size.ravel(), [0.0]]))
        np.testing.assert_array_equal(np.isnan(gm), np.isnan(want))
        assert not np.nanmax(np.abs(gm - want) - (2.0 ** -18 + dm) * want) > 1e-37
    return out, m


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_store_and_read_are_exact(layout, dtype):
    hq, hkv, hd = layout
    p = Pair(layout, dtype, 100, 3, lengths=[100, 37, 16], seed=3, scale=3.0)
    k, v = p.cache.read(0, 3, 100, lengths=_ints(p.lengths))
    for b, m in enumerate(p.lengths):
        np.testing.assert_array_equal(_np(k)[b, :, :m], p.held.k[b, :, :m])
        np.testing.assert_array_equal(_np(v)[b, :, :m], p.held.v[b, :, :m])
        assert (_np(k)[b, :, m:] == 0).all() and (_np(v)[b, :, m:] == 0).all()
    k2, v2 = p.cache.read(0, 3, 20, firsts=_ints([5, 30, 0]), lengths=_ints(p.lengths))
    np.testing.assert_array_equal(_np(k2)[0], p.held.k[0, :, 5:25])
    np.testing.assert_array_equal(_np(v2)[1, :, :7], p.held.v[1, :, 30:37])
    assert (_np(k2)[1, :, 7:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_appending_behind_tokens_raises_the_block_exponents(dtype):
    p = Pair((4, 2, 72), dtype, 64, 2, lengths=[21, 0])
    starts, scale = [21, 0], 1.0
    for n in (1, 1, 3, 15, 1):          # within blocks, across them, ever larger values
        scale *= 5.0
        k, v = _rand((2, n, 2, 72), n, dtype, scale), _rand((2, n, 2, 72), 90 + n, dtype, 1 / scale)
        p.cache.append(0, k, v, _ints(starts))
        p.held.append(_np(k), _np(v), starts, [n, n])
        starts = [s + n for s in starts]
    k, v = p.cache.read(0, 2, 64, lengths=_ints(starts))
    for b, m in enumerate(starts):
        np.testing.assert_array_equal(_np(k)[b, :, :m], p.held.k[b, :, :m])
        np.testing.assert_array_equal(_np(v)[b, :, :m], p.held.v[b, :, :m])


def test_extreme_values_are_held_as_defined():
    p = Pair((1, 1, 16), "fp32", 64, 1)
    k = torch.zeros((1, 48, 1, 16), device="cuda")
    k[0, 0] = 3e38
    k[0, 1] = 1e-38
    k[0, 16] = 1e-45
    k[0, 17] = 448 * 2.0 ** -100
    k[0, 32, 0, 3] = 448.0
    k[0, 33, 0, 4] = -0.0
    k[0, 34, 0, 5] = float(np.nextafter(np.float32(448), np.float32(500)))
    v = -k.flip(1)
    p.cache.append(0, k, v)
    p.held.append(_np(k), _np(v), [0], [48])
    gk, gv = p.cache.read(0, 1, 48)
    np.testing.assert_array_equal(_np(gk)[0], p.held.k[0, :, :48])
    np.testing.assert_array_equal(_np(gv)[0], p.held.v[0, :, :48])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("tokens", [1, 15, 64, 333])
def test_single_tokens(layout, dtype, tokens):
    p = Pair(layout, dtype, tokens + 5, 2, lengths=[tokens, max(1, tokens // 3)], seed=tokens)
    check(p, 1, mass=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", [(8, 1, 256), (16, 4, 64), (6, 2, 40), (4, 4, 128), (5, 1, 192)])
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 1, 0), (True, 33, 5), (True, 70, 17)])
def test_runs_of_queries(layout, dtype, causal, window, sinks):
    p = Pair(layout, dtype, 260, 3, queries=37, lengths=[256, 131, 40])
    check(p, 37, causal=causal, window=window, sinks=sinks, mass=True)
    check(p, 37, counts=[37, 5, 0], causal=causal, window=window, sinks=sinks, mass=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout,n", [((8, 1, 256), 150), ((16, 4, 64), 201), ((4, 4, 128), 260), ((6, 2, 40), 130), ((3, 1, 192), 100)])
@pytest.mark.parametrize("causal,window,sinks", [(False, 0, 0), (True, 0, 0), (True, 50, 4)])
def test_prompts(layout, n, dtype, causal, window, sinks):
    p = Pair(layout, dtype, n + 9, 2, queries=n, lengths=[n + 9, n - 63], seed=n)
    check(p, n, counts=[n, n - 90], causal=causal, window=window, sinks=sinks, mass=True)


def test_robots_without_tokens_or_queries_get_zeros():
    p = Pair((8, 2, 64), "bf16", 64, 3, queries=4, lengths=[0, 20, 3])
    out, m = check(p, 4, counts=[0, 0, 3], mass=True)
    assert (_np(out)[:2] == 0).all() and (_np(out)[2, 3] == 0).all() and (_np(m)[:2] == 0).all()
    p.lengths = [0, 0, 0]
    out, m = check(p, 4, counts=[0, 0, 0], causal=False, mass=True)
    assert (_np(out) == 0).all() and (_np(m) == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [1, 40])
def test_what_is_not_finite_reaches_only_those_that_see_it(dtype, n):
    p = Pair((8, 2, 64), dtype, 160, 2, queries=n, lengths=[150, 150])
    k, v = _rand((2, 1, 2, 64), 50, dtype), _rand((2, 1, 2, 64), 51, dtype)
    k[0, 0, 1, 7] = float("inf")
    v[1, 0, 0, 3] = float("nan")
    starts = [120, 100]     # a token in the past of the last queries, outside a window of 20
    p.cache.append(0, k, v, _ints(starts))
    p.held.append(_np(k), _np(v), starts, [1, 1])
    # (what lay behind it in its block is stored again)
    k, v = _rand((2, 60, 2, 64), 52, dtype), _rand((2, 60, 2, 64), 53, dtype)
    starts = [121, 101]
    cnt = [29, 49]
    p.cache.append(0, k, v, _ints(starts), counts=_ints(cnt))
    p.held.append(_np(k), _np(v), starts, cnt)
    out, m = check(p, n, mass=True)
    assert np.isnan(_np(out)).any() and np.isfinite(_np(out)).any()
    out, m = check(p, n, window=20, sinks=3, mass=True)
    assert np.isfinite(_np(out)[:, -1]).all()
    q = _rand((2, n, 8, 64), 60, dtype)
    q[0, 0, 2, 5] = float("inf")
    q[1, n - 1, 7, 0] = float("nan")
    p2 = Pair((8, 2, 64), dtype, 160, 2, queries=n, lengths=[150, 90])
    out = p2.cache.attend(0, q, _ints(p2.lengths))
    bad = torch.isnan(out).cpu().numpy()
    want = np.zeros(bad.shape, bool)
    want[0, 0, 2] = want[1, n - 1, 7] = True
    np.testing.assert_array_equal(bad, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [1, 20])
def test_peaked_and_flat_rows_and_values_of_many_sizes(dtype, n):
    """Scores up to a few hundred, blocks of values 2^20 apart, robots that differ."""
    p = Pair((4, 2, 64), dtype, 200, 2, queries=n)
    p.lengths = [200, 77]
    k, v = _rand((2, 200, 2, 64), 1, dtype), _rand((2, 200, 2, 64), 2, dtype)
    v = v * (2.0 ** (torch.arange(200, device="cuda") // 16 % 5 * 5 - 10)).to(v.dtype)[None, :, None, None]
    p.cache.append(0, k, v, counts=_ints(p.lengths))
    p.held.append(_np(k), _np(v), [0, 0], p.lengths)
    for q_scale in (1e-6, 0.1, 30.0):
        check(p, n, q_scale=q_scale, mass=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_long_flat_tail_keeps_its_weight(dtype):
    """One token far above 20000 flat ones whose weight together is that of the one."""
    T, hd = 20000, 64
    p = Pair((1, 1, hd), dtype, T, 1)
    p.lengths = [T]
    k = torch.zeros((1, T, 1, hd), device="cuda")
    k[0, 5, 0, 0] = 8.0
    v = torch.ones((1, T, 1, hd), device="cuda")
    v[0, 5] = 0.0
    q = torch.zeros((1, 1, 1, hd), device="cuda")
    q[0, 0, 0, 0] = 10.0             # score 10 against 0: weight 22026 to 19999
    k, v, q = (x.to(_dt(dtype)) for x in (k, v, q))
    p.cache.append(0, k, v)
    p.held.append(_np(k), _np(v), [0], [T])
    check(p, 1, q=q, mass=True)


def test_strided_unaligned_and_layered_tensors():
    """q, k, v as columns of one projection, at offsets that allow no wide loads, in layer 2 of 3."""
    from paper_2609_34170_gb300 import ContextCache
    for hq, hkv, hd, dtype, off in ((8, 2, 64, "bf16", 0), (6, 2, 40, "bf16", 3), (6, 2, 40, "fp32", 1)):
        B, n = 2, 19
        rows = _rand((B, n + 2, (hq + 2 * hkv) * hd + 5), 1, dtype)
        cut = [rows[:, 1:n + 1, off + a * hd:off + (a + w) * hd].unflatten(2, (w, hd))
               for a, w in ((0, hq), (hq, hkv), (hq + hkv, hkv))]
        c = ContextCache(3, hq, hkv, hd, 64, B, n, dtype)
        c.append(2, cut[1], cut[2])
        out = torch.full((B, n, hq * hd + 7), 9.0, dtype=_dt(dtype), device="cuda")
        view = out[:, :, 1:1 + hq * hd].unflatten(2, (hq, hd))
        c.attend(2, cut[0], _ints([n, n]), out=view)
        c2 = ContextCache(1, hq, hkv, hd, 64, B, n, dtype)
        c2.append(0, cut[1].contiguous(), cut[2].contiguous())
        want = c2.attend(0, cut[0].contiguous(), _ints([n, n]))
        assert torch.equal(view, want)
        assert (out[:, :, 0] == 9.0).all() and (out[:, :, 1 + hq * hd:] == 9.0).all()
        for layer in (0, 1):
            assert (c.read(layer, B, 64)[0] == 0).all()


def test_mass_adds_up_and_repeats_bit_for_bit():
    p = Pair((8, 1, 256), "bf16", 700, 2, queries=3, lengths=[700, 411])
    q = _rand((2, 3, 8, 256), 5, "bf16")
    L = _ints(p.lengths)
    m1 = torch.empty((2, 1, 700), device="cuda")
    o1 = p.cache.attend(0, q, L, mass=m1)
    m2 = m1.clone()
    o2 = p.cache.attend(0, q, L, mass=m2, add_mass=True)
    assert torch.equal(o1, o2)
    assert torch.equal(m2, m1 + m1)
    assert torch.allclose(m1.sum(-1), torch.full((2, 1), 24.0, device="cuda"), rtol=1e-5)
    for _ in range(3):
        m3 = torch.empty_like(m1)
        assert torch.equal(p.cache.attend(0, q, L, mass=m3), o1) and torch.equal(m3, m1)


@pytest.mark.parametrize("layout,n,batch", [((8, 1, 256), 300, 16), ((8, 2, 128), 300, 10), ((8, 1, 64), 300, 16), ((8, 1, 192), 300, 16)])
def test_prompts_of_many_robots_repeat_bit_for_bit(layout, n, batch):
    # more row tiles than SMs: their second ones start while the first ones' output is written
    p = Pair(layout, "bf16", n + 12, batch, queries=n, lengths=[n + 3 * (b % 5) for b in range(batch)], seed=21)
    q = _rand((batch, n, layout[0], layout[2]), 22, "bf16", 2.0)
    first, _ = check(p, n, q=q)
    first = first.clone()
    for _ in range(40):
        out = p.cache.attend(0, q, _ints(p.lengths))
        assert torch.equal(out, first)


def test_other_streams_scales_and_bounds():
    p = Pair((16, 4, 64), "bf16", 300, 2, queries=2, lengths=[300, 200])
    q = _rand((2, 2, 16, 64), 5, "bf16")
    L = _ints(p.lengths)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    want = p.cache.attend(0, q, L, scale=0.125)
    torch.cuda.synchronize()
    got = p.cache.attend(0, q, L, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    out = torch.empty_like(q)
    with torch.cuda.graph(g):
        p.cache.attend(0, q, L, out=out)
    L.copy_(_ints([10, 5]))       # lengths are read when the graph runs
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, p.cache.attend(0, q, _ints([10, 5])))
    assert torch.equal(out, p.cache.attend(0, q, _ints([10, 5]), max_length=10)) or \
        torch.allclose(out.float(), p.cache.attend(0, q, _ints([10, 5]), max_length=10).float(), rtol=2 ** -7)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", [(8, 1, 256), (16, 4, 64), (6, 2, 40)])
@pytest.mark.parametrize("keep,sinks,recent", [(64, 4, 16), (33, 0, 0), (20, 4, 16), (500, 0, 7), (1, 0, 1)])
def test_eviction(layout, dtype, keep, sinks, recent):
    from paper_2609_34170_gb300 import ContextCache
    hq, hkv, hd = layout
    lengths = [333, 70, 20]
    p = Pair(layout, dtype, 333, 3, lengths=lengths, scale=2.0)
    rng = np.random.default_rng(4)
    mass = rng.integers(0, 12, (3, hkv, 340)).astype(np.float32) / 3     # many ties
    mass[0, :, 100:110] = np.inf
    mass[0, 0, 50] = np.nan
    mass[0, 0, 60:64] = -0.0
    mass[0, 0, 64] = -1.5
    to = ContextCache(2, hq, hkv, hd, keep, 3, 1, dtype)
    got = p.cache.evict(0, to, 1, _ints(lengths), torch.from_numpy(mass).cuda(), keep, sinks, recent)
    k, v = to.read(1, 3, keep, lengths=got[0])
    n, index, kept, held = ref.evict(p.held, lengths, mass, keep, sinks, recent)
    np.testing.assert_array_equal(got[0].cpu().numpy(), n)
    np.testing.assert_array_equal(got[1].cpu().numpy(), index)
    np.testing.assert_array_equal(_np(got[2]), kept)
    np.testing.assert_array_equal(_np(k), held.k[:, :, :keep])
    np.testing.assert_array_equal(_np(v), held.v[:, :, :keep])


def test_eviction_from_long_caches():
    from paper_2609_34170_gb300 import ContextCache
    T, keep = 40000, 3001
    p = Pair((4, 1, 64), "bf16", T, 1, lengths=[T])
    mass = np.random.default_rng(1).random((1, 1, T)).astype(np.float32) ** 4
    to = ContextCache(1, 4, 1, 64, keep, 1, 1, "bf16")
    got = p.cache.evict(0, to, 0, _ints([T]), torch.from_numpy(mass).cuda(), keep, 4, 100)
    n, index, kept, held = ref.evict(p.held, [T], mass, keep, 4, 100)
    np.testing.assert_array_equal(got[1].cpu().numpy(), index)
    k, _ = to.read(0, 1, keep)
    np.testing.assert_array_equal(_np(k), held.k[:, :, :keep])


@pytest.mark.parametrize("layout,n,batch", [((16, 4, 64), 900, 3), ((3, 3, 40), 150, 130), ((16, 1, 64), 1100, 1)])
def test_mass_whose_scores_come_in_parts(layout, n, batch):
    # more scores than are kept at a time: some robots', then some queries'
    p = Pair(layout, "fp32", n + 40, batch, queries=n, lengths=[n + 40 - 7 * (b % 5) for b in range(batch)], seed=41)
    check(p, n, mass=True, counts=[n - b % 3 for b in range(batch)])
    _, m = check(p, n, mass=True, causal=False, seed=9)
    q = _rand((batch, n, layout[0], layout[2]), 9, "fp32", 2.0)
    twice = m.clone()
    p.cache.attend(0, q, _ints(p.lengths), causal=False, mass=twice, add_mass=True)
    for b, length in enumerate(p.lengths):
        torch.testing.assert_close(twice[b, :, :length], 2 * m[b, :, :length], rtol=2 ** -20, atol=0)
        assert torch.equal(twice[b, :, length:], m[b, :, length:])


def _chain(cache, small, x, lengths, n):
    """Append, attend with the mass, evict and read back, none of them waited for."""
    cache.append(0, x["k"], x["v"])
    out = cache.attend(0, x["q"], lengths, mass=x["mass"])
    kept, index, mass = cache.evict(0, small, 0, lengths, x["mass"], 50, sinks=2, recent=5)
    return (out, x["mass"]) + (kept, index, mass) + small.read(0, x["k"].shape[0], 50, lengths=kept)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout,n", [((8, 1, 256), 1), ((8, 1, 256), 40), ((16, 4, 64), 70)])
def test_chained_calls_wait_for_each_other(layout, n, dtype):
    # launches may start before the ones before them have ended: what one writes the next reads
    from paper_2609_34170_gb300 import ContextCache
    hq, hkv, hd = layout
    batch, tokens = 5, 300
    lengths = _ints([300, 200, 120, 299, 250])
    xs = []
    for i in range(6):
        xs.append({"k": _rand((batch, tokens, hkv, hd), 50 + i, dtype), "v": _rand((batch, tokens, hkv, hd), 60 + i, dtype),
                   "q": _rand((batch, n, hq, hd), 70 + i, dtype, 2.0), "mass": torch.zeros((batch, hkv, tokens), device="cuda")})
    cache, small = ContextCache(1, hq, hkv, hd, tokens, batch, n, dtype), ContextCache(1, hq, hkv, hd, 64, batch, 1, dtype)
    want = []
    for x in xs:
        got = _chain(cache, small, x, lengths, n)
        torch.cuda.synchronize()
        want.append([t.clone() for t in got])
    for x in xs:
        x["mass"].fill_(-1.0)
    torch.cuda.synchronize()
    for _ in range(5):
        got = [_chain(cache, small, x, lengths, n) for x in xs]
        for a, b in zip(got, want):
            for t, w in zip(a, b):
                assert torch.equal(t, w)


@pytest.mark.parametrize("n", [1, 40])
def test_calls_replay_from_a_graph(n):
    from paper_2609_34170_gb300 import ContextCache
    batch, tokens = 3, 200
    cache, small = ContextCache(1, 8, 1, 256, tokens, batch, n), ContextCache(1, 8, 1, 256, 64, batch, 1)
    lengths = _ints([200, 77, 150])
    x = {"k": _rand((batch, tokens, 1, 256), 80, "bf16"), "v": _rand((batch, tokens, 1, 256), 81, "bf16"),
         "q": _rand((batch, n, 8, 256), 82, "bf16", 2.0), "mass": torch.zeros((batch, 1, tokens), device="cuda")}
    _chain(cache, small, x, lengths, n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = _chain(cache, small, x, lengths, n)
    for seed in (83, 93):
        for i, name in enumerate(("k", "v", "q")):
            x[name].copy_(_rand(x[name].shape, seed + i, "bf16"))
        lengths.copy_(_ints([seed, 200, 60]))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        want = _chain(cache, small, x, lengths, n)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_refusals():
    from paper_2609_34170_gb300 import ContextCache, RavelError
    p = Pair((4, 2, 64), "bf16", 64, 2, queries=4, lengths=[30, 20])
    c, q, L = p.cache, _rand((2, 4, 4, 64), 1, "bf16"), _ints([30, 20])
    k = _rand((2, 3, 2, 64), 1, "bf16")

    def refused(status, call):
        with pytest.raises(RavelError) as ei:
            call()
        assert ei.value.status == status, str(ei.value)

    refused(1, lambda: c.attend(0, q, L, causal=False, window=3))
    refused(1, lambda: c.attend(0, q, L, sinks=3))
    refused(1, lambda: c.attend(0, q, L, window=-1))
    refused(1, lambda: c.attend(0, q, L, scale=-1.0))
    refused(1, lambda: c.attend(0, q, L, scale=float("nan")))
    refused(2, lambda: c.attend(1, q, L))
    refused(2, lambda: c.attend(0, q, L, max_length=65))
    refused(2, lambda: c.attend(0, _rand((2, 5, 4, 64), 1, "bf16"), L))
    refused(2, lambda: c.attend(0, _rand((3, 4, 4, 64), 1, "bf16"), _ints([1, 1, 1])))
    refused(2, lambda: c.attend(0, q, L, mass=torch.zeros((2, 2, 63), device="cuda")))
    refused(2, lambda: c.append(0, _rand((2, 65, 2, 64), 1, "bf16"), _rand((2, 65, 2, 64), 1, "bf16")))
    refused(2, lambda: c.read(0, 2, 129))
    to = ContextCache(1, 4, 2, 64, 32, 2, 1)
    mass = torch.zeros((2, 2, 64), device="cuda")
    refused(1, lambda: c.evict(0, c, 0, L, mass, 8))
    refused(2, lambda: c.evict(0, to, 0, L, mass, 33))
    refused(2, lambda: c.evict(0, to, 0, L, mass, 8, sinks=4, recent=5))
    refused(2, lambda: c.evict(0, to, 1, L, mass, 8))
    for call in (lambda: c.attend(0, q.float(), L), lambda: c.attend(0, q, L.long()), lambda: c.attend(0, q, _ints([1])),
                 lambda: c.attend(0, q.transpose(1, 2), L), lambda: c.attend(0, q, L, mass=mass[:1]),
                 lambda: c.append(0, k.float(), k.float()), lambda: c.append(0, k, k.transpose(2, 3)),
                 lambda: c.append(0, k, k[:, :2])):
        with pytest.raises(ValueError):
            call()
    # values of the device arrays: the robot is left out, a later call reports it
    want = c.attend(0, q, L)
    for bad, cnt in (([65, 20], None), ([-1, 20], None), ([3, 20], None), ([30, 20], [5, 4]), ([30, 20], [-1, 4])):
        out = c.attend(0, q, _ints(bad), counts=None if cnt is None else _ints(cnt))
        torch.cuda.synchronize()
        assert (out[0] == 0).all() and torch.equal(out[1], want[1])
        refused(7, lambda: c.attend(0, q, L))
        c.reset()
    for starts, cnt in (([62, 0], None), ([-1, 0], None), ([0, 0], [4, 0]), ([0, 0], [-1, 0])):
        before = c.read(0, 2, 64)[0]
        c.append(0, k, k, _ints(starts), counts=_ints(cnt or [3, 0]))
        torch.cuda.synchronize()
        refused(7, lambda: c.attend(0, q, L))
        c.reset()
        if cnt is None:
            assert torch.equal(c.read(0, 2, 64)[0][0], before[0])
    p.cache.evict(0, to, 0, _ints([65, 20]), mass, 8)
    torch.cuda.synchronize()
    refused(7, lambda: c.read(0, 2, 4))
    c.reset()
    c.read(0, 2, 4, firsts=_ints([-1, 0]))
    torch.cuda.synchronize()
    refused(7, lambda: c.read(0, 2, 4))
    c.reset()
    assert torch.equal(c.attend(0, q, L), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_calls_on_a_handle_do_what_the_class_does(dtype):
    import paper_2609_34170_gb300 as pkg
    batch, n, hq, hkv, hd, keep = 2, 21, 6, 2, 40, 13
    k, v = _rand((batch, 30, hkv, hd), 1, dtype), _rand((batch, 30, hkv, hd), 2, dtype)
    q, lengths = _rand((batch, n, hq, hd), 3, dtype, 2.0), _ints([30, 22])
    cache, small = (pkg.ContextCache(2, hq, hkv, hd, t, batch, n, dtype) for t in (40, keep))
    cache.append(1, k, v, counts=lengths)
    mass = torch.zeros((batch, hkv, 40), device="cuda")
    want = [cache.attend(1, q, lengths, window=9, sinks=2, mass=mass), mass]
    want += cache.evict(1, small, 0, lengths, mass, keep, 2, 3)
    want += small.read(0, batch, keep, lengths=want[2])
    kind = pkg.RAVEL_BF16 if dtype == "bf16" else pkg.RAVEL_FP32
    c, to = (pkg.ravel_cache_create(2, hq, hkv, hd, t, batch, n, kind) for t in (40, keep))
    try:
        got = [torch.empty_like(t) for t in want]
        pkg.ravel_cache_append(c, 1, k, v, counts=lengths)
        pkg.ravel_cache_attend(c, 1, q, got[0], lengths, None, 40, window=9, sinks=2, mass=got[1])
        pkg.ravel_cache_evict(c, 1, to, 0, lengths, got[1], keep, 2, 3, got[2], got[3], got[4])
        pkg.ravel_cache_read(to, 0, got[5], got[6], lengths=got[2])
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    finally:
        torch.cuda.synchronize()
        pkg.ravel_cache_destroy(c)
        pkg.ravel_cache_destroy(to)


def test_a_cache_refused_for_want_of_memory_leaves_the_library_usable():
    """The runtime keeps a failed call's error until it is asked for; the step's launches ask."""
    import synth
    from paper_2609_34170_gb300 import ContextCache, RavelError
    from tests._harness import Case, check_step, gpu_session
    case = Case(synth.ExpertConfig(layers=1, width=192, n_q_heads=6, n_kv_heads=2, head_dim=40, mlp_dim=320, slots=7, action_dim=5,
                                   prefix=45, fop_tokens=3, batch=2, dtype="bf16"))
    session = gpu_session(case)
    for turn in range(2):
        with pytest.raises(RavelError) as ei:
            ContextCache(1024, 8, 4, 256, 1 << 20, 4)      # 1 TB of keys
        assert ei.value.status == 3
        session.reset(case.seeds)
        if turn:                                           # (the session came with one)
            session.set_context(case.k, case.v, case.P)
        check_step(case, session)
    session.close()
    p = Pair((8, 2, 64), "bf16", 64, 2, queries=4, lengths=[30, 20])
    check(p, 4, mass=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_eviction_keeps_the_largest_finite_values(dtype):
    """What is held as 2^128, which neither type has, is no infinity on its way to another cache."""
    from paper_2609_34170_gb300 import ContextCache
    info = torch.finfo(_dt(dtype))
    p = Pair((2, 2, 24), dtype, 64, 1)
    k, v = _rand((1, 60, 2, 24), 1, dtype), _rand((1, 60, 2, 24), 2, dtype)
    k[0, 3, 0, 5] = info.min
    k[0, 40, 1, 0] = info.max
    v[0, 3, 1, 7], v[0, 21, 0, 2] = info.max, 3.2e38
    v[0, 22, 0, 1], k[0, 23, 0, 0] = info.tiny, 2.0 ** -100
    p.cache.append(0, k, v)
    p.held.append(_np(k), _np(v), [0], [60])
    mass = np.random.default_rng(3).random((1, 2, 64)).astype(np.float32)
    mass[:, :, [3, 21, 22, 23, 40]] = 2.0
    cache, held, lengths = p.cache, p.held, [60]
    for keep in (37, 17):         # out of the first cache, and out of the second again
        to = ContextCache(1, 2, 2, 24, keep, 1, 1, dtype)
        got = cache.evict(0, to, 0, _ints(lengths), torch.from_numpy(mass).cuda(), keep, 2, 3)
        lengths, index, mass64, held = ref.evict(held, lengths, mass, keep, 2, 3)
        np.testing.assert_array_equal(got[1].cpu().numpy(), index)
        for g, w in zip(to.read(0, 1, keep, lengths=got[0]), (held.k, held.v)):
            with np.errstate(over="ignore"):
                np.testing.assert_array_equal(_np(g), w[:, :, :keep].astype(np.float32).astype(np.float64))
        cache, mass, lengths = to, mass64.astype(np.float32), list(lengths)


def test_a_decoded_token_whose_key_and_value_lie_apart():
    from paper_2609_34170_gb300 import ContextCache
    c, want = (ContextCache(1, 4, 2, 64, 32, 1, 1) for _ in range(2))
    qkv = _rand((1, 1, 8, 64), 1, "bf16")
    q, k, v = qkv[:, :, :4], _rand((1, 1, 2, 64), 4, "bf16"), qkv[:, :, 6:]
    assert k.stride() != v.stride()
    for cache in (c, want):
        cache.append(0, _rand((1, 9, 2, 64), 2, "bf16"), _rand((1, 9, 2, 64), 3, "bf16"))
    c.append(0, k, v, _ints([9]))
    want.append(0, k, torch.empty_like(k).copy_(v), _ints([9]))
    for a, b in zip(c.read(0, 1, 10), want.read(0, 1, 10)):
        assert torch.equal(a, b)
    out = torch.empty((1, 3, 4, 64), dtype=torch.bfloat16, device="cuda")[:, 1:2]
    assert torch.equal(c.attend(0, q, _ints([10]), out=out), want.attend(0, torch.empty((1, 1, 4, 64), dtype=q.dtype, device="cuda").copy_(q), _ints([10])))


def _within(pair, got, q, n, causal=True, window=0, sinks=0, mass=None, counts=None):
    """bf16 attention of many rows against the reference, with a score's error as it is there: 2^-18
    of scale sum |q k| for the sums, and each element of q off by up to 2^-21 of the row's largest;
    scores off by d change weights by a factor of up to e^2d."""
    counts = [n] * pair.batch if counts is None else counts
    o, ms, W, size = ref.attend(_np(q), pair.held, pair.lengths, counts, causal, window, sinks)
    hq, hkv, hd = pair.layout
    keys = np.abs(pair.held.k).sum(-1).max(-1).repeat(hq // hkv, 1)            # [B, Hq]: the largest sum of |k|
    d = 2.0 ** -18 * size + 2.0 ** -21 / np.sqrt(hd) * np.abs(_np(q)).max(-1) * keys[:, None]
    tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -10 + np.expm1(2 * d[..., None])) * W
    err = np.abs(_np(got) - o)
    assert (err <= tol + 1e-37).all(), (err.max(), (err / (tol + 1e-37)).max())
    if mass is not None:
        m = _np(mass)[:, :, :ms.shape[2]]
        ms = ms[:, :, :m.shape[2]]
        assert (np.abs(m - ms) <= (2.0 ** -18 + np.expm1(2 * d.max())) * ms + 1e-37).all()


@pytest.mark.parametrize("layout,n", [((2, 1, 40), 20), ((4, 1, 64), 40), ((2, 2, 128), 140), ((3, 1, 192), 30), ((8, 1, 256), 5)])
@pytest.mark.parametrize("big", [2.0 ** 7, 2.0 ** 12, 2.0 ** 15])
def test_small_dims_beside_a_large_one_keep_their_weight(layout, n, big):
    """A query's first dim is far above the others, and the keys do not use it."""
    hq, hkv, hd = layout
    p = Pair(layout, "bf16", 300, 2, queries=n)
    p.lengths = [300, 201]
    rng = np.random.default_rng(1)
    sign = rng.choice([-1.0, -0.5, 0.5, 1.0], (2, 300, hkv, 1))
    for same in (True, False):        # dims that add up, and dims of any size
        k = np.ones((2, 300, hkv, hd)) * sign if same else rng.standard_normal((2, 300, hkv, hd))
        k[..., 0] = 0.0
        # (just below half a unit of what e4m3 holds beside the largest)
        q = np.full((2, n, hq, hd), 0.97) if same else 2.0 ** rng.uniform(-12, 6, (2, n, hq, hd)) * rng.choice([-1, 1], (2, n, hq, hd))
        q *= 2.0 ** -17 * big
        q[..., 0] = big
        k, q = (torch.from_numpy(x).to(torch.bfloat16).cuda() for x in (k, q))
        v = _rand((2, 300, hkv, hd), 2, "bf16")
        p.cache.append(0, k, v, counts=_ints(p.lengths))
        p.held.append(_np(k), _np(v), [0, 0], p.lengths)
        for causal, window, sinks in ((False, 0, 0), (True, 60, 4)):
            mass = torch.zeros((2, hkv, 300), device="cuda")
            out = p.cache.attend(0, q, _ints(p.lengths), causal=causal, window=window, sinks=sinks, mass=mass)
            _within(p, out, q, n, causal, window, sinks, mass)
