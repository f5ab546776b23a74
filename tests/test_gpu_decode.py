"""Rotary positions, 4-bit products and drawing tokens on the GPU against 64-bit references.

Rotary: a turned value is own c - other s (fp32).  c and s are off by at most 2^-24 (the angle, at most
pi / 4, in fp32) + 2^-24 (one unit of the function at 1) + 2^-25 (the amplitude), the product and the sum
add 2 x 2^-24: below 2^-21 (|x| + |y|) amplitude.  The frequency's own 2^-52 is position f 2^-51 on top.
Then half a step of the type, 2^-8 |result| in bf16.

Products: exact terms x (c - z) are summed on the tensor core in chains of up to eight MMAs.  Each keeps its 17
addends to 24 bits below the largest, which for the spread values here is below a quarter of the group's sum of
magnitudes: 8 x 16 x 2^-24 / 4 = 2^-19 of it; the scale and the sums over the groups (at most two per 64 ks, then 8
warps and 8 ranks) add 2^-24 each: (2^-19 + (K / 32 + 18) 2^-24) sum |x w|.  Then the epilogue and the output's half step.

Tokens are equal; log-probabilities within 2^-23 of their size and 1e-7."""
import math

import numpy as np
import pytest

from oracle import cache as cache_ref
from oracle import decode as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_34170_gb300 import build, load
    build.build()
    load()


def _dt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _rand(shape, seed, dtype="fp32", scale=1.0):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape) * scale).to(_dt(dtype)).cuda()


def _ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _f32(x):
    return torch.tensor(np.asarray(x), dtype=torch.float32, device="cuda")


def _np(t):
    return t.detach().double().cpu().numpy()


def _half(dtype):
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24


# ---- rotary positions

TURNS = [(64, 64, False), (256, 256, False), (256, 256, True), (64, 32, False), (40, 40, False), (40, 24, True), (128, 34, True),
         (256, 2, False), (72, 18, False), (6, 6, True), (7, 4, False), (80, 80, False), (80, 48, True), (64, 16, False), (2, 2, True)]


def _turn_close(got, x, positions, f, dims, interleaved, dtype, amplitude=1.0):
    want = ref.turn(x, positions, f, interleaved, amplitude)
    size = ref.pair_size(x, dims, interleaved) * abs(amplitude)
    far = np.abs(np.asarray(positions, np.float64)).max() * np.abs(f).max() * 2.0 ** -51
    tol = (2.0 ** -21 + far) * size + _half(dtype) * np.abs(want) * (size > 0)
    assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) - tol)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd,dims,interleaved", TURNS)
def test_turns_heads(hd, dims, interleaved, dtype):
    from paper_2609_34170_gb300 import Rotary
    r = Rotary(dims, interleaved=interleaved, base=5e5, amplitude=1.25)
    f = ref.frequencies(dims, base=5e5)
    for batch, n, heads in ((3, 5, 3), (1, 1, 1), (2, 70, 9)):
        x = _rand((batch, n, heads, hd), hd + n, dtype)
        starts = np.array([0, 37, 1000003][:batch])
        got = r.apply(x, starts=_ints(starts))
        _turn_close(_np(got), _np(x), starts[:, None] + np.arange(n), f, dims, interleaved, dtype, 1.25)
        assert torch.equal(got[..., dims:], x[..., dims:])
        y = x.clone()
        assert r.apply(y, starts=_ints(starts), out=y) is y and torch.equal(y, got)   # in place


def test_turns_columns_of_a_projection_and_leaves_the_rest():
    from paper_2609_34170_gb300 import Rotary
    qkv = _rand((2, 9, 6, 64), 3, "bf16")
    keep = qkv.clone()
    r = Rotary(64)
    pos = np.random.default_rng(0).integers(-5000, 5000, (2, 9))
    heads = qkv[:, :, :5]
    r.apply(heads, positions=_ints(pos), counts=_ints([4, -3]), out=heads)
    _turn_close(_np(qkv)[:1, :4, :5], _np(keep)[:1, :4, :5], pos[:1, :4], ref.frequencies(64), 64, False, "bf16")
    assert torch.equal(qkv[0, 4:], keep[0, 4:]) and torch.equal(qkv[1], keep[1]) and torch.equal(qkv[:, :, 5], keep[:, :, 5])
    out = torch.full((2, 9, 5, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    r.apply(keep[:, :, :5], positions=_ints(pos), counts=_ints([2, 99]), out=out)   # a count past n is n
    assert (out[0, 2:] == 7).all() and not (out[1] == 7).all()
    new = r.apply(keep[:, :, :5], positions=_ints(pos), counts=_ints([2, 0]))
    assert (new[0, 2:] == 0).all() and (new[1] == 0).all() and torch.equal(new[0, :2], out[0, :2])


@pytest.mark.parametrize("dtype,offset,dims", [("bf16", 1, 64), ("bf16", 4, 64), ("fp32", 1, 32), ("fp32", 2, 64)])
def test_turns_unaligned_rows(dtype, offset, dims):
    from paper_2609_34170_gb300 import Rotary
    flat = _rand((3 * 4 * 2 * 64 + 200,), 5, dtype)
    x = flat[offset:].as_strided((3, 4, 2, 64), (4 * 133, 133, 64, 1))
    r = Rotary(dims)
    a, b = r.apply(x), r.apply(x.contiguous())
    assert torch.equal(a, b)


def test_turns_far_positions():
    """In float angles half of these are noise."""
    from paper_2609_34170_gb300 import Rotary
    x = _rand((1, 6, 2, 64), 8)
    pos = np.array([[-2 ** 31, -123456789, 0, 10 ** 7, 2 ** 30 + 1, 2 ** 31 - 1]])
    _turn_close(_np(Rotary(64).apply(x, positions=_ints(pos))), _np(x), pos, ref.frequencies(64), 64, False, "fp32")
    start = Rotary(64).apply(x[:, :1], starts=_ints([2 ** 31 - 1]))
    assert torch.equal(start, Rotary(64).apply(x[:, :1], positions=_ints([[2 ** 31 - 1]])))


def test_turns_by_stretched_and_given_frequencies():
    from paper_2609_34170_gb300 import Rotary
    x = _rand((1, 3, 2, 64), 9)
    pos = np.array([[5, 4000, 30000]])
    settings = dict(base=1e4, factor=8.0, original_length=2048.0, low=2.0, high=16.0)
    f = ref.frequencies(64, **settings)
    _turn_close(_np(Rotary(64, **settings).apply(x, positions=_ints(pos))), _np(x), pos, f, 64, False, "fp32")
    _turn_close(_np(Rotary(64, factor=4.0).apply(x, positions=_ints(pos))), _np(x), pos, ref.frequencies(64) / 4, 64, False, "fp32")
    own = np.linspace(-3.0, 9.0, 32)
    _turn_close(_np(Rotary(64, frequencies=own).apply(x, positions=_ints(pos))), _np(x), pos, own, 64, False, "fp32")


def test_the_transpose_is_the_turn_to_the_negative_position():
    """<R x, y> = <x, R(-p) y>: its rounding is 2^-21 of the sums of magnitudes on either side."""
    from paper_2609_34170_gb300 import Rotary
    r = Rotary(48, interleaved=True, amplitude=0.5)
    x, y = _rand((2, 7, 3, 64), 10), _rand((2, 7, 3, 64), 11)
    pos = np.random.default_rng(1).integers(0, 10000, (2, 7))
    a = (_np(r.apply(x, positions=_ints(pos))) * _np(y)).sum()
    b = (_np(x) * _np(r.apply(y, positions=_ints(-pos)))).sum()
    assert abs(a - b) <= 2.0 ** -20 * 2 * (np.abs(_np(x)).sum() + 1) * np.abs(_np(y)).max()


def test_turning_nothing_is_nothing():
    from paper_2609_34170_gb300 import Rotary
    r = Rotary(16)
    for shape in ((0, 3, 2, 16), (2, 0, 2, 16), (2, 3, 0, 16)):
        assert r.apply(torch.empty(shape, device="cuda")).shape == shape


def test_rotary_refusals():
    from paper_2609_34170_gb300 import RavelError, Rotary
    r = Rotary(32)
    with pytest.raises(RavelError):   # heads smaller than the table
        r.apply(torch.zeros((1, 1, 1, 16), device="cuda"))
    x = torch.zeros((2, 4, 1, 32), device="cuda")
    with pytest.raises(RavelError):   # in place with other strides
        r.apply(x[:, :2], out=x.as_strided((2, 2, 1, 32), (64, 32, 32, 1)))


# ---- stores with rotation


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout,dims,interleaved", [((8, 1, 256), 256, False), ((16, 4, 64), 64, True), ((6, 2, 40), 40, False),
                                                     ((6, 2, 40), 16, True), ((4, 4, 128), 34, False), ((3, 1, 72), 64, False),
                                                     ((20, 1, 64), 64, False), ((1, 1, 8), 8, False), ((5, 1, 192), 96, True)])
def test_append_rotary_is_apply_then_append(layout, dims, interleaved, dtype):
    """Bit for bit, with fp32 between the two; queries as apply gives them."""
    from paper_2609_34170_gb300 import ContextCache, Rotary
    hq, hkv, hd = layout
    r = Rotary(dims, interleaved=interleaved)
    cache = ContextCache(1, hq, hkv, hd, 100, 3, 1, dtype)
    plain = ContextCache(1, hq, hkv, hd, 100, 3, 1, "fp32")
    first = [_rand((3, 16, hkv, hd), s, dtype) for s in (1, 2)]
    cache.append(0, *first, starts=_ints([16, 32, 0]))
    plain.append(0, *(t.float() for t in first), starts=_ints([16, 32, 0]))
    for n, starts, counts in ((1, [21, 47, 0], None), (37, [30, 33, 5], [37, 0, 21]), (16, [0, 64, 7], None)):
        qkv = _rand((3, n, hq + 2 * hkv, hd), n, dtype, 2.0)
        q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
        pos = _ints(np.random.default_rng(n).integers(0, 200000, (3, n))) if n != 16 else None
        c = None if counts is None else _ints(counts)
        got = cache.append_rotary(0, r, q, k, v, _ints(starts), counts=c, positions=pos)
        turned = r.apply(k.float(), starts=_ints(starts), positions=pos)
        plain.append(0, turned.contiguous(), v.float().contiguous(), _ints(starts), counts=c)
        assert torch.equal(got, r.apply(q, starts=_ints(starts), positions=pos, counts=c))
        for a, b in zip(cache.read(0, 3, 100), plain.read(0, 3, 100)):
            assert torch.equal(a.float(), b)
        cache.append_rotary(0, r, q, k, v, _ints(starts), counts=c, positions=pos, q_out=q)   # queries in place
        assert torch.equal(q, got if counts is None else torch.where((torch.arange(n, device="cuda")[None] < c[:, None])[..., None, None], got, q))


def test_append_rotary_against_the_reference():
    """Held keys against the reference's rounding of keys turned in 64 bits: equal but where fp32's error
    (2^-21 of a pair) crosses a rounding border, where they differ by one step (2^-3 of the value, 2^-9 of the block's unit)."""
    from paper_2609_34170_gb300 import ContextCache, Rotary
    hq, hkv, hd = 8, 2, 64
    k, v = _rand((2, 50, hkv, hd), 5, "bf16"), _rand((2, 50, hkv, hd), 6, "bf16")
    cache = ContextCache(1, hq, hkv, hd, 64, 2)
    pos = np.arange(50)[None] + np.array([[0], [70000]])
    assert cache.append_rotary(0, Rotary(hd), None, k, v, positions=_ints(pos)) is None
    held = cache_ref.Held(2, hkv, 64, hd)
    held.append(ref.turn(_np(k), pos, ref.frequencies(hd)), _np(v), [0, 0], [50, 50])
    gk, gv = (_np(t) for t in cache.read(0, 2, 50))
    np.testing.assert_array_equal(gv, held.v[:, :, :50])
    want = held.k[:, :, :50]
    assert (np.abs(gk - want) <= 2.0 ** -3 * np.abs(want) + 2.0 ** -9).all() and (gk != want).mean() < 1e-3


def test_append_rotary_reports_positions_out_of_range():
    from paper_2609_34170_gb300 import ContextCache, RavelError, Rotary
    cache = ContextCache(1, 2, 1, 64, 32, 2)
    k, q = _rand((2, 4, 1, 64), 0, "bf16"), _rand((2, 4, 2, 64), 1, "bf16")
    out = torch.full_like(q, 3.0)
    cache.append_rotary(0, Rotary(64), q, k, k, _ints([30, 0]), q_out=out)
    torch.cuda.synchronize()
    assert (out[0] == 3).all() and not (out[1] == 3).all()
    cache.reset()
    k20, q20 = _rand((2, 20, 1, 64), 0, "bf16"), _rand((2, 20, 2, 64), 1, "bf16")
    for starts, counts in (([13, 0], None), ([-1, 0], None), ([0, 0], [21, 20]), ([0, 0], [-1, 20]), ([30, 0], [3, 20])):
        out20 = torch.full_like(q20, 3.0)
        cache.append_rotary(0, Rotary(64), q20, k20, k20, _ints(starts), counts=None if counts is None else _ints(counts), q_out=out20)
        torch.cuda.synchronize()
        assert (out20[0] == 3).all() and not (out20[1] == 3).any()
        cache.reset()
    cache = ContextCache(1, 2, 1, 64, 32, 2)
    cache.append_rotary(0, Rotary(64), q, k, k, _ints([30, 0]), q_out=out)
    torch.cuda.synchronize()
    with pytest.raises(RavelError) as ei:
        cache.append_rotary(0, Rotary(64), q, k, k, _ints([0, 0]))
    assert ei.value.status == 7
    cache.reset()
    assert (cache.read(0, 2, 32)[0][0] == 0).all()
    with pytest.raises(RavelError):   # more dims than a head
        ContextCache(1, 2, 1, 32, 32, 2).append_rotary(0, Rotary(64), None, k[..., :32].contiguous(), k[..., :32].contiguous())


# ---- 4-bit products


def _weights(n, k, group, seed):
    rng = np.random.default_rng(seed)
    groups = -(-k // group)
    codes = rng.integers(0, 16, (n, k), dtype=np.uint8)
    scales = ref.bf16(rng.uniform(-1, 2, (n, groups)) / math.sqrt(k))
    zeros = rng.integers(0, 16, (n, groups), dtype=np.uint8)
    return codes, scales, zeros


def _held(n, k, group, seed=0):
    from paper_2609_34170_gb300 import Weights4
    codes, scales, zeros = _weights(n, k, group, seed)
    packed = ref.pack(codes)
    if k % 2:   # the last high nibble means nothing
        packed[:, -1] |= 0xF0
    w = Weights4(n, k, group)
    w.load(torch.from_numpy(packed).cuda(), torch.from_numpy(scales).to(torch.bfloat16).cuda(), torch.from_numpy(zeros).cuda())
    return w, ref.weights(packed, scales, zeros, k, group)


def _product_close(got, x, w, epi, out_dtype, bias=None, before=None):
    y = x @ w.T + (0 if bias is None else bias)
    err = (2.0 ** -19 + (w.shape[1] / 32 + 18) * 2.0 ** -24) * (np.abs(x) @ np.abs(w).T) + 2.0 ** -23 * np.abs(y)
    if epi == "silu":
        want = y / (1 + np.exp(-y))
        err = 1.1 * err + 2.0 ** -21 * np.abs(want)
    elif epi == "geglu":
        (g, u), (eg, eu) = ref.geglu_rows(y), ref.geglu_rows(err)
        want = ref.gelu(g) * u
        # tanh is off by 2^-22 at most, half of it times g
        err = (1.13 * eg + 2.0 ** -22 * np.abs(g)) * (np.abs(u) + eu) + np.abs(ref.gelu(g)) * eu + 2.0 ** -22 * np.abs(want)
    elif epi == "add":
        want = y + before
        err = err + 2.0 ** -24 * np.abs(want)
    else:
        want = y
    tol = err + _half(out_dtype) * (np.abs(want) + err) + 1e-37
    assert np.isfinite(got).all() and (np.abs(got - want) <= tol).all(), np.max((np.abs(got - want) - tol) / tol)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,k", [(1, 1), (16, 64), (31, 40), (33, 130), (77, 1003), (640, 1024), (128, 4096), (1000, 520)])
def test_products(n, k, group):
    w, held = _held(n, k, group, n + k)
    np.testing.assert_array_equal(_np(w.read(torch.float32)), held.astype(np.float32))
    np.testing.assert_array_equal(_np(w.read()), ref.bf16(held.astype(np.float32)))
    bias = _rand((n,), 3)
    for m in (1, 2, 7, 8, 9, 16, 17, 32, 33, 64, 65, 130):
        x = _rand((m, k), m, "bf16")
        for epi, dtype, b in (("store", "bf16", None), ("silu", "fp32", bias), ("add", "fp32", None), ("store", "fp32", bias)):
            before = _rand((m, n), m + 1)
            out = before.clone() if epi == "add" else torch.empty((m, n), dtype=_dt(dtype), device="cuda")
            got = w.product(x, out=out, epi=epi, bias=b)
            assert got is out
            _product_close(_np(got), _np(x), held, epi, dtype, None if b is None else _np(b), _np(before))
            if m > 16:
                break


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,k", [(4113, 70), (5000, 1003), (4097, 2056), (9000, 512), (17000, 1000), (700, 20000)])
def test_products_of_many_rows_of_weights(n, k, group):
    """Where pairs of tiles share the tokens' values: ends inside a tile, a stage, a group and a cluster's share."""
    w, held = _held(n, k, group, n)
    flat = _rand((130 * (k + 16),), 1, "bf16")
    up = -(-k // 8) * 8
    for m, lda, offset in ((17, up, 0), (32, k + 1, 0), (33, up, 0), (64, up + 8, 8), (70, k, 1), (129, up, 16)):
        x = flat[offset:].as_strided((m, k), (lda, 1))
        bias = _rand((n,), 3)
        _product_close(_np(w.product(x, dtype=torch.float32, bias=bias)), _np(x), held, "store", "fp32", _np(bias))
    before = _rand((129, n), 2)
    _product_close(_np(w.product(x, out=before.clone(), epi="add")), _np(x), held, "add", "fp32", None, _np(before))


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("n,k", [(128, 64), (384, 333), (8192, 1024), (4224, 1500), (16384, 1096)])
def test_geglu_products(n, k, group):
    w, held = _held(n, k, group, n)
    bias = _rand((n,), 4)
    for m in (1, 4, 12, 32, 50, 72, 200):
        x = _rand((m, k), m, "bf16")
        _product_close(_np(w.product(x, epi="geglu")), _np(x), held, "geglu", "bf16")
        _product_close(_np(w.product(x, epi="geglu", bias=bias)), _np(x), held, "geglu", "bf16", _np(bias))


@pytest.mark.parametrize("group", [32, 64, 128])
def test_products_whose_last_round_is_shared(group):
    """More tiles than SMs, and few in the last round: pairs of CTAs share those, every epilogue."""
    w, held = _held(20480, 1100, group, 5)
    flat, bias = _rand((70, 1104), 1, "bf16"), _rand((20480,), 4)
    for m in (31, 58, 70):
        x = flat[:m, :1100]
        _product_close(_np(w.product(x, epi="geglu", bias=bias)), _np(x), held, "geglu", "bf16", _np(bias))
        _product_close(_np(w.product(x, epi="silu", dtype=torch.float32)), _np(x), held, "silu", "fp32")
        before = _rand((m, 20480), 2)
        _product_close(_np(w.product(x, out=before.clone(), epi="add", bias=bias)), _np(x), held, "add", "fp32", _np(bias), _np(before))
    w, held = _held(20449, 1101, group, 6)
    x = flat[:33, :1101]
    _product_close(_np(w.product(x)), _np(x), held, "store", "bf16")


def test_products_of_strided_and_unaligned_rows_touch_nothing_else():
    w, held = _held(50, 104, 32)
    flat = _rand((20 * 131 + 40,), 5, "bf16")
    for offset, lda in ((0, 112), (8, 120), (1, 131), (0, 131)):
        x = flat[offset:].as_strided((20, 104), (lda, 1))
        out = torch.full((20, 61), -5.0, device="cuda")
        w.product(x, out=out[:, 3:53])
        _product_close(_np(out[:, 3:53]), _np(x), held, "store", "fp32")
        assert (out[:, :3] == -5).all() and (out[:, 53:] == -5).all()


def test_values_that_are_not_finite_stay_in_their_rows():
    w, held = _held(40, 100, 32)
    x = _rand((5, 104), 6, "bf16")
    x[:, 100:] = float("nan")     # columns behind K are no part of it
    x[2, 50] = float("inf")
    x[3, 1] = float("nan")
    got = _np(w.product(x[:, :100], dtype=torch.float32))
    rows = [0, 1, 4]
    _product_close(got[rows], _np(x)[rows, :100], held, "store", "fp32")
    assert not np.isfinite(got[2]).all() and np.isnan(got[3]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_quantises_to_the_nearest_codes(dtype):
    from paper_2609_34170_gb300 import Weights4
    from paper_2609_34170_gb300.decode import quantize4
    w = _rand((37, 205), 7, dtype, 0.02)
    w[3] = 0
    w[4, :64] = w[4, :64].abs()
    w[5, :64] = -w[5, :64].abs()
    for group in (32, 64, 128):
        codes, scales, zeros = quantize4(w[:, :203], group)
        c, s, z = ref.quantize(_np(w)[:, :203].astype(np.float32), group)
        np.testing.assert_array_equal(_np(scales), s)
        np.testing.assert_array_equal(zeros.cpu().numpy(), z)
        np.testing.assert_array_equal(codes.cpu().numpy(), ref.pack(c))
        held = Weights4.quantize(w[:, :203], group).read(torch.float32)
        np.testing.assert_array_equal(_np(held), ref.weights(ref.pack(c), s, z, 203, group).astype(np.float32))


def test_quantises_the_largest_and_smallest_values():
    """Groups whose values lie further apart than fp32 reaches, and whose scale is bf16's smallest or none."""
    from paper_2609_34170_gb300.decode import Weights4, quantize4
    w = torch.zeros((4, 64), device="cuda")
    w[0, :2] = torch.tensor([3e38, -3e38])
    w[1, :2] = torch.tensor([3e38, -1e38])   # (beyond 3e38 the nearest code's value may be beyond fp32: excluded)
    w[2, :2] = torch.tensor([2.0 ** -130, -2.0 ** -131])
    w[3, :2] = torch.tensor([2.0 ** -140, 0.0])
    held = _np(Weights4.quantize(w, 32).read(torch.float32))
    step = np.array([6e38, 4e38, 1.5 * 2.0 ** -130, 2.0 ** -140]) / 15
    # half a step where codes round, 0.04 for the zero point's rounding and the scale's 2^-9 of 15 steps at the ends,
    # and a scale below bf16's smallest, 2^-133, moves by up to half of that, 15 times
    assert (np.abs(held - _np(w)) <= 1.04 * step[:, None] + np.array([0, 0, 7.5, 7.5])[:, None] * 2.0 ** -133).all()
    assert torch.isfinite(quantize4(w, 32)[1]).all()


def test_overlapping_rows_are_refused():
    from paper_2609_34170_gb300 import RavelError, Rotary
    r = Rotary(16)
    x = _rand((1, 5, 2, 32), 0, "bf16").expand(3, 5, 2, 32)
    assert (r.apply(x)[2] == r.apply(x)[0]).all()   # reading the same rows is fine
    for out in (x, torch.empty_strided((3, 5, 2, 32), (64, 64, 32, 1), dtype=torch.bfloat16, device="cuda")):
        with pytest.raises(RavelError) as ei:
            r.apply(x, out=out)
        assert ei.value.status == 1


def test_product_refusals():
    from paper_2609_34170_gb300 import RavelError, Weights4
    w = Weights4(96, 64, 32)
    assert (w.read() == 0).all()
    x = _rand((2, 64), 0, "bf16")
    assert (w.product(x) == 0).all()
    assert w.product(x[:0]).shape == (0, 96)
    with pytest.raises(RavelError):   # rows are no blocks of 128
        w.product(x, epi="geglu")
    with pytest.raises(RavelError):   # adds to fp32
        w.product(x, epi="add", out=torch.zeros((2, 96), dtype=torch.bfloat16, device="cuda"))
    for bad in (dict(epi="relu"), dict(epi="add")):
        with pytest.raises(ValueError):
            w.product(x, **bad)
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    codes, scales, zeros = torch.zeros((96, 32), dtype=torch.uint8, device="cuda"), torch.ones((96, 2), dtype=torch.bfloat16, device="cuda"), \
        torch.zeros((96, 2), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        with pytest.raises(RavelError) as ei:   # loading waits: not under capture
            w.load(codes, scales, zeros)
        w.product(x)
    assert ei.value.status == 1


# ---- drawing tokens


def _draws(x, u, t=None, k=None, p=None, q=None):
    from paper_2609_34170_gb300 import draw_tokens
    b = len(u)
    got, logs = draw_tokens(x, _f32(u), *(None if s is None else _f32(s) for s in (t,)), top_k=None if k is None else _ints(k),
                            top_p=None if p is None else _f32(p), min_p=None if q is None else _f32(q), log_probs=True)
    got, logs, rows = got.cpu().numpy(), _np(logs), _np(x)
    f = np.float32
    for i in range(b):
        token, log = ref.draw(rows[i], f(u[i]), f(1.0 if t is None else t[i]), 0 if k is None else int(k[i]), f(1.0 if p is None else p[i]),
                              f(0.0 if q is None else q[i]))
        assert got[i] == token, (i, got[i], token)
        assert logs[i] == log or abs(logs[i] - log) <= 2.0 ** -23 * abs(log) + 1e-7, (i, logs[i], log)
    return got


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 33, 257, 4099, 32003, 65536, 151000])
def test_draws_under_every_mix_of_limits(vocab, dtype):
    rng = np.random.default_rng(vocab)
    mixes = [(1.0, 0, 1.0, 0.0), (0.7, 40, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.3, 0, 1.0, 0.05), (0.8, 50, 0.95, 0.02), (1.0, 3, 0.2, 0.9),
             (2.5, 1000, 0.99, 0.0), (0.05, 5, 0.5, 0.1), (0.0, 9, 0.4, 0.0), (1.0, vocab, 0.5, 0.0), (1.0, 1, 1.0, 0.0), (1.0, -4, 2.0, -1.0),
             (1.0, 0, 0.0, 0.0), (1.0, 0, -0.5, 5.0), (1e-7, 0, 0.5, 0.0), (50.0, 0, 0.999, 0.0), (1.0, 20, 0.999999, 1e-4)]
    b = len(mixes)
    t, k, p, q = zip(*mixes)
    for scale in (3.0, 0.1):
        x = _rand((b, vocab), vocab + 1, dtype, scale)
        for u in (rng.random(b, dtype=np.float32), np.zeros(b), np.full(b, 1 - 2.0 ** -24)):
            _draws(x, u, t, k, p, q)


@pytest.mark.parametrize("vocab", [64, 1500, 40000])
def test_draws_among_ties_by_index(vocab):
    """Equal logits: sums of equal weights, limits in the middle of them."""
    u = np.array([0.0, 0.25, 0.5, 0.999, 0.3, 0.8])
    flat = torch.zeros((6, vocab), device="cuda")
    for p, k in ((None, None), ([0.5] * 6, None), (None, [vocab // 3] * 6), ([0.25] * 6, [vocab // 2] * 6)):
        _draws(flat, u, p=p, k=k)
    steps = (torch.arange(vocab, device="cuda")[None] * 7 % 5).float().repeat(6, 1)
    for p, k in ((None, [vocab // 4] * 6), ([0.7] * 6, None), ([0.9] * 6, [vocab // 2 + 1] * 6)):
        _draws(steps, u, p=p, k=k)
    signs = torch.where(torch.arange(vocab, device="cuda")[None] % 2 == 0, 0.0, -0.0).repeat(6, 1)   # -0 is 0
    _draws(signs, u, k=[vocab // 2] * 6)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab,spread", [(20000, 3.0), (20000, 0.01), (100003, 1.0), (1 << 20, 2.0)])
def test_draws_where_more_stays_than_a_list_holds(vocab, spread, dtype):
    """Limits of thousands of tokens, alone and together, and rows so flat that one bin of the order holds thousands."""
    mixes = [(1.0, 3000, 1.0, 0.0), (1.0, 3000, 0.9, 0.0), (1.0, 3000, 1.0, 0.001), (0.9, 9000, 0.999, 1e-5), (1.0, 0, 0.97, 0.0),
             (1.0, 0, 0.97, 0.01), (1.0, 2047, 0.5, 0.0), (1.0, 2048, 1.0, 0.0), (3.0, 2049, 0.7, 0.0), (1.0, 0, 0.999999, 0.0)]
    x = _rand((len(mixes), vocab), vocab, dtype, spread)
    t, k, p, q = zip(*mixes)
    for seed in range(3):
        _draws(x, np.random.default_rng(seed).random(len(mixes), dtype=np.float32), t, k, p, q)


def test_masks_and_rows_that_cannot_be_drawn_from():
    x = _rand((9, 5000), 1, "fp32", 3.0)
    inf, nan = math.inf, math.nan
    hide = torch.rand((5000,), device="cuda") < 0.99
    x[0, hide] = -inf
    x[1] = -inf
    x[1, 4321] = -300.0
    x[2] = -inf
    x[3, 17] = nan
    x[4, 18] = inf
    x[5] = torch.finfo(torch.float32).min
    x[6] = -1e30
    x[6, 77] = 3e38
    x[7, ::2] = torch.finfo(torch.float32).min
    x[8] = 3e38
    got = _draws(x, np.full(9, 0.5), k=[0, 3, 0, 0, 0, 2, 0, 0, 0], p=[0.9] * 9)
    assert (got[[2, 3, 4]] == -1).all() and got[1] == 4321 and got[6] == 77
    y = _rand((10, 300), 2)
    one = [1.0] * 10
    got = _draws(y, [nan, -0.1, 1.0, inf, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5], one[:4] + [nan, inf, -inf, 1.0, 1.0, -2.0], p=one[:7] + [nan] + one[8:],
                 q=[0.0] * 8 + [nan, 0.0])
    assert (got[[0, 1, 2, 3, 4, 5, 7, 8]] == -1).all() and (got[[6, 9]] >= 0).all()


def test_a_spread_of_the_whole_range_does_not_overflow():
    x = _rand((3, 1000), 3) * 1e38
    x[:, 0], x[:, 1] = 3.4e38, -3.4e38
    _draws(x, [0.1, 0.5, 0.9], t=[1e38, 3e38, 1e37], p=[0.9, 1.0, 0.99])


@pytest.mark.parametrize("dtype,offset,stride", [("bf16", 1, 1031), ("bf16", 0, 1040), ("fp32", 3, 1033), ("fp32", 0, 1028)])
def test_draws_from_strided_and_unaligned_rows(dtype, offset, stride):
    flat = _rand((9 * 1040 + 8,), 4, dtype, 3.0)
    flat[-1] = math.nan
    x = flat[offset:].as_strided((7, 1021), (stride, 1))
    _draws(x, np.linspace(0, 0.99, 7), k=[30] * 7, p=[0.9] * 7)


def test_many_rows_and_repeats():
    from paper_2609_34170_gb300 import draw_tokens
    rng = np.random.default_rng(0)
    x, u = _rand((700, 1500), 5, "bf16", 2.0), rng.random(700, dtype=np.float32)
    first = _draws(x, u, p=[0.8] * 700)
    for _ in range(3):
        assert (draw_tokens(x, _f32(u), top_p=_f32([0.8] * 700)).cpu().numpy() == first).all()
    assert draw_tokens(x[:0], _f32([])).shape == (0,)


def test_draws_follow_their_distribution():
    """Evenly spread u give each token its share of the draws to one in their number."""
    n = 4000
    logits = torch.tensor([1.0, -2.0, 0.5, 3.0, -math.inf, 0.0], device="cuda")
    from paper_2609_34170_gb300 import draw_tokens
    got = draw_tokens(logits.repeat(n, 1), (torch.arange(n, device="cuda") + 0.5) / n).cpu().numpy()
    share = np.exp(_np(logits)) / np.exp(_np(logits)).sum()
    assert (np.abs(np.bincount(got, minlength=6) - n * share) <= 1.01).all()


# ---- together


def _step(m, tokens, u, lengths, counts):
    """One decoded token per robot: every operator behind the other, as a program calls them."""
    from paper_2609_34170_gb300 import draw_tokens
    x = m["embed"][tokens.long()]
    qkv = m["qkv"].product(x).unflatten(-1, (1, m["hq"] + 2 * m["hkv"], m["hd"]))
    hq, hkv = m["hq"], m["hkv"]
    q = m["cache"].append_rotary(0, m["rotary"], qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:], lengths, positions=m["pos"])
    att = m["cache"].attend(0, q, lengths + counts, max_length=64)
    res = x.float()
    m["o"].product(att.flatten(1), out=res, epi="add")
    hidden = m["up"].product(res.to(torch.bfloat16), epi="geglu")
    m["down"].product(hidden, out=res, epi="add")
    logits = m["head"].product(res.to(torch.bfloat16), dtype=torch.float32)
    return (qkv, q, att, res, hidden, logits) + draw_tokens(logits, u, top_k=m["k"], top_p=m["p"], log_probs=True)


def _model(batch):
    from paper_2609_34170_gb300 import ContextCache, Rotary
    hq, hkv, hd, d, f, vocab = 4, 2, 64, 256, 512, 1000
    m = dict(hq=hq, hkv=hkv, hd=hd, embed=_rand((vocab, d), 1, "bf16"), rotary=Rotary(hd), cache=ContextCache(1, hq, hkv, hd, 64, batch))
    for name, n, k in (("qkv", (hq + 2 * hkv) * hd, d), ("o", d, hq * hd), ("up", 2 * f, d), ("down", d, f), ("head", vocab, d)):
        m[name], m[name + "64"] = _held(n, k, 64, n)
    m["cache"].append(0, _rand((batch, 20, hkv, hd), 2, "bf16"), _rand((batch, 20, hkv, hd), 3, "bf16"))
    m["k"], m["p"], m["pos"] = _ints([50] * batch), _f32([0.9] * batch), _ints([[100 + 7 * b] for b in range(batch)])
    return m


def test_a_decoded_token_goes_through_all_of_them():
    batch = 5
    m = _model(batch)
    lengths, one = _ints([20, 3, 17, 9, 1]), _ints([1] * batch)
    tokens, u = _ints([5, 900, 33, 0, 999]), _f32(np.random.default_rng(3).random(batch))
    qkv, q, att, res, hidden, logits, drawn, logs = _step(m, tokens, u, lengths, one)
    x = _np(m["embed"])[tokens.cpu().numpy()]
    _product_close(_np(qkv).reshape(batch, -1), x, m["qkv64"], "store", "bf16")
    _turn_close(_np(q), _np(qkv)[:, :, :4], m["pos"].cpu().numpy(), ref.frequencies(64), 64, False, "bf16")
    mid = x + _np(att).reshape(batch, -1) @ m["o64"].T
    gate, up = ref.geglu_rows(mid @ m["up64"].T)
    want = ref.gelu(gate) * up
    assert np.linalg.norm(_np(hidden) - want) <= 2.0 ** -6 * np.linalg.norm(want)   # (mid is rounded to bf16 on the way)
    _product_close(_np(logits), _np(res.to(torch.bfloat16)), m["head64"], "store", "fp32")
    for b in range(batch):
        assert int(drawn[b]) == ref.draw(_np(logits)[b], np.float32(u[b].item()), 1.0, 50, np.float32(0.9))[0]


def test_replayed_and_chained_steps_equal_eager_ones():
    """Launches that begin while the one before ends: 12 steps without a wait between them, eager and from a graph."""
    batch, steps = 5, 12
    us = _f32(np.random.default_rng(4).random((steps, batch)))
    one = _ints([1] * batch)

    def run(graphed):
        m = _model(batch)
        lengths, tokens, u = _ints([20] * batch), _ints([1, 2, 3, 4, 5]), us[0].clone()
        out = []

        def step():
            drawn = _step(m, tokens, u, lengths, one)[-2]
            tokens.copy_(drawn)
            lengths.add_(1)

        if graphed:
            step()
            lengths.fill_(20)
            tokens.copy_(_ints([1, 2, 3, 4, 5]))
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        for i in range(steps):
            u.copy_(us[i])
            graph.replay() if graphed else step()
            out.append(tokens.clone())
        torch.cuda.synchronize()
        return torch.stack(out)

    eager = run(False)
    assert torch.equal(eager, run(False)) and torch.equal(eager, run(True))


FIRST_CALLS = """
import sys; sys.path.insert(0, sys.argv[1])
import torch
from paper_2609_34170_gb300 import Rotary, Weights4, draw_tokens
w, r = Weights4(4200, 512, 64), Rotary(32)
x = torch.randn((40, 512), device="cuda").to(torch.bfloat16)
u, starts = torch.full((40,), 0.5, device="cuda"), torch.arange(40, dtype=torch.int32, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = w.product(x), r.apply(x.view(40, 1, 16, 32), starts=starts), draw_tokens(x, u), w.product(x[:5]), draw_tokens(x.float(), u)
graph.replay()
torch.cuda.synchronize()
again = w.product(x), r.apply(x.view(40, 1, 16, 32), starts=starts), draw_tokens(x, u), w.product(x[:5]), draw_tokens(x.float(), u)
assert all(torch.equal(a, b) for a, b in zip(got, again))
print("the same")
"""


def test_first_calls_may_be_captured():
    """In a process of its own, where nothing has run before the capture."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", FIRST_CALLS, root], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "the same" in done.stdout, done.stderr[-2000:]


def test_a_matrix_can_be_reset_and_loaded_again():
    from paper_2609_34170_gb300 import Weights4
    x = _rand((3, 96), 0, "bf16")
    w = Weights4(40, 96, 32)
    for seed in (1, 2):
        codes, scales, zeros = _weights(40, 96, 32, seed)
        w.load(torch.from_numpy(ref.pack(codes)).cuda(), torch.from_numpy(scales).to(torch.bfloat16).cuda(), torch.from_numpy(zeros).cuda())
        w.reset()
        _product_close(_np(w.product(x, dtype=torch.float32)), _np(x), ref.weights(ref.pack(codes), scales, zeros, 96, 32), "store", "fp32")
    w.close()
    with pytest.raises(ValueError):
        w.product(x)


def test_two_streams_share_weights_and_a_table():
    from paper_2609_34170_gb300 import Rotary, draw_tokens
    w, _ = _held(512, 1024, 64)
    r = Rotary(64)
    xs = [_rand((4, 1024), s, "bf16") for s in (1, 2)]
    want = [(w.product(x, dtype=torch.float32), r.apply(x.view(4, 1, 16, 64), starts=_ints([9] * 4)),
             draw_tokens(x, _f32([0.3] * 4))) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    starts, u = _ints([9] * 4), _f32([0.3] * 4)
    torch.cuda.synchronize()
    got = []
    for i in range(40):
        x, s = xs[i % 2], streams[i % 2]
        got.append((w.product(x, dtype=torch.float32, stream=s), r.apply(x.view(4, 1, 16, 64), starts=starts, stream=s.cuda_stream),
                    draw_tokens(x, u, stream=s)))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[i % 2]))
