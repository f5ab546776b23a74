"""Rotary positions, 4-bit products and drawing tokens without a GPU: the 64-bit
references against closed forms, and what is refused before a device is touched."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import decode as ref
from tests.test_cache_host import _Gpu as _Cache

torch = pytest.importorskip("torch")


class _Gpu(_Cache):
    """Stands in for a CUDA tensor: all that the calls look at, none of the memory."""

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        return self._stride if i is None else self._stride[i]


@pytest.fixture(scope="module")
def lib():
    from paper_2609_34170_gb300 import build, load
    build.build()
    return load()


def test_reference_turns():
    f = ref.frequencies(4, base=100.0)
    np.testing.assert_allclose(f, [1.0, 0.1])
    x = np.zeros((1, 1, 1, 6))
    x[..., 0], x[..., 5] = 1.0, 7.0
    y = ref.turn(x, [[2]], f)
    np.testing.assert_allclose(y[0, 0, 0], [math.cos(2), 0, math.sin(2), 0, 0, 7])
    y = ref.turn(x, [[2]], f, interleaved=True)
    np.testing.assert_allclose(y[0, 0, 0], [math.cos(2), math.sin(2), 0, 0, 0, 7])


def test_reference_frequencies_between_the_borders():
    f = ref.frequencies(64, base=1e4)
    g = ref.frequencies(64, base=1e4, factor=8.0, original_length=4096)
    turns = 4096 * f / (2 * math.pi)
    np.testing.assert_array_equal(g[turns >= 32], f[turns >= 32])
    np.testing.assert_allclose(g[turns <= 1], f[turns <= 1] / 8)
    assert ((g <= f) & (g >= f / 8)).all() and (np.diff(g) < 0).all()


def test_reference_scores_depend_on_distances_only():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 1, 1, 32))
    f = ref.frequencies(32)
    scores = [(ref.turn(q, [[p + 17]], f) * ref.turn(k, [[p]], f)).sum() for p in (0, 5, 123456)]
    np.testing.assert_allclose(scores, scores[0], atol=1e-9)


def test_reference_quantises_to_nearest():
    rng = np.random.default_rng(1)
    w = rng.standard_normal((5, 100)).astype(np.float32)
    w[2] = 0
    codes, s, z = ref.quantize(w, 32)
    held = ref.weights(ref.pack(codes), s, z, 100, 32)
    assert s.shape == z.shape == (5, 4)
    # within half a step of the group, and the zero point's rounding at the ends
    assert (np.abs(held - w) <= s[:, np.arange(100) // 32] * 1.07).all()
    assert (held[2] == 0).all()
    np.testing.assert_array_equal(ref.unpack(ref.pack(codes), 100), codes)


def test_reference_draws():
    x = np.log([0.1, 0.4, 0.2, 0.3])
    assert [ref.draw(x, u)[0] for u in (0.0, 0.05, 0.2, 0.6, 0.8)] == [0, 0, 1, 2, 3]
    assert ref.draw(x, 0.99, top_k=2)[0] == 3 and ref.draw(x, 0.5, top_k=2)[0] == 1
    assert ref.draw(x, 0.99, top_p=0.65)[0] == 3 and ref.draw(x, 0.99, top_p=0.39)[0] == 1
    assert ref.draw(x, 0.0, min_p=0.6)[0] == 1 and ref.draw(x, 0.0, min_p=0.45)[0] == 1
    assert ref.draw(x, 0.9, temperature=0.0) == (1, 0.0)
    assert abs(ref.draw(x, 0.0, top_k=2)[1] - math.log(4 / 7)) < 1e-12
    assert ref.draw([1.0, 1.0, 1.0], 0.9, top_k=1)[0] == 0
    assert ref.draw([-np.inf, np.nan], 0.5) == ref.draw([-np.inf], 0.5) == ref.draw([np.inf, 0], 0.5) == (-1, -math.inf)


def test_null_arguments_are_refused(lib):
    n = None
    assert lib.ravel_rotary_create(n, 0, n) == 1
    assert lib.ravel_rotary_apply(n, 1, 1, 1, 8, 0, n, 0, 0, n, 0, 0, n, n, n, n) == 1
    assert lib.ravel_cache_append_rotary(n, 0, n, 1, 1, n, 0, 0, n, 0, 0, n, 0, 0, n, 0, 0, n, n, n, n) == 1
    assert lib.ravel_w4_create(1, 1, 32, 0, n) == 1
    assert lib.ravel_w4_load(n, n, n, n, n) == 1
    assert lib.ravel_w4_quantize(n, 1, 1, 1, 0, 32, n, n, n, n) == 1
    assert lib.ravel_w4_read(n, n, 1, 0, n) == 1
    assert lib.ravel_w4_reset(n) == 1
    assert lib.ravel_w4_gemm(n, n, 1, 1, 0, n, 1, 0, n, n) == 1
    assert lib.ravel_draw_tokens(n, 1, 1, 1, 0, n, n, n, n, n, n, n, n) == 1
    assert b"draw_tokens" in lib.ravel_decode_last_error()
    lib.ravel_rotary_destroy(n)
    lib.ravel_w4_destroy(n)


def test_rotary_refuses_settings(lib):
    from paper_2609_34170_gb300 import RavelError, ravel_rotary_create
    for bad in (dict(dims=0), dict(dims=7), dict(dims=258), dict(base=0.0), dict(base=-1.0), dict(base=math.inf), dict(factor=0.0),
                dict(factor=math.nan), dict(original_length=-1.0), dict(original_length=64.0, low=4.0, high=4.0),
                dict(original_length=64.0, low=-1.0), dict(amplitude=math.inf), dict(frequencies=[math.nan] * 8)):
        with pytest.raises(RavelError) as ei:
            ravel_rotary_create(**{**dict(dims=16), **bad})
        assert ei.value.status == 1
    with pytest.raises(ValueError):
        ravel_rotary_create(16, frequencies=[1.0] * 7)


def test_matrices_and_rows_of_impossible_sizes_are_refused(lib):
    from paper_2609_34170_gb300 import RavelError, ravel_w4_create
    for args, status in (((8, 8, 48), 1), ((0, 8, 32), 2), ((8, 0, 32), 2), (((1 << 24) + 1, 8, 32), 2)):
        with pytest.raises(RavelError) as ei:
            ravel_w4_create(*args)
        assert ei.value.status == status
    p = C.c_void_p(256)
    assert lib.ravel_draw_tokens(p, 1, 0, 1, 0, p, None, None, None, None, p, None, None) == 2
    assert lib.ravel_draw_tokens(p, 1, (1 << 20) + 1, 1 << 21, 0, p, None, None, None, None, p, None, None) == 2
    assert lib.ravel_draw_tokens(p, 2, 8, 7, 0, p, None, None, None, None, p, None, None) == 2
    assert lib.ravel_draw_tokens(p, 1, 8, 8, 2, p, None, None, None, None, p, None, None) == 1
    assert lib.ravel_draw_tokens(p, 0, 8, 8, 0, p, None, None, None, None, p, None, None) == 0   # no row: nothing to do
    assert lib.ravel_w4_quantize(p, 8, 8, 7, 0, 32, p, p, p, None) == 2


def _rotary_handle():
    r = C.c_void_p()
    r.rotary = (16, 0)
    return r


def test_rotary_refuses_tensors_that_do_not_fit(lib):
    import paper_2609_34170_gb300 as pkg
    from paper_2609_34170_gb300 import _binding as B
    b16, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    r = _rotary_handle()
    x, ints, pos = _Gpu((3, 5, 2, 32), b16), _Gpu((3,), i32), _Gpu((3, 5), i32)

    def apply(r=r, x=x, out=None, **more):
        pkg.ravel_rotary_apply(r, x, out or x, **{**dict(starts=ints, positions=pos, counts=ints), **more}, stream=0)

    with pytest.raises(B.RavelError):   # what fits goes to the library, whose handle is null
        apply()
    with pytest.raises(ValueError):
        apply(r=C.c_void_p())
    for bad in (_Gpu((3, 5, 64), b16), _Gpu((3, 5, 2, 32), b16, device=1), _Gpu((3, 5, 2, 32), torch.float16),
                _Gpu((3, 5, 2, 32), b16, (320, 64, 32, 2)), _Gpu((3, 5, 2, 32), b16, (640, 128, 64, 1))):
        with pytest.raises(ValueError):
            apply(x=bad)
    for bad in (_Gpu((3, 5, 2, 32), f32), _Gpu((3, 4, 2, 32), b16)):
        with pytest.raises(ValueError):
            apply(out=bad)
    for name, bad in (("starts", _Gpu((2,), i32)), ("starts", _Gpu((3,), f32)), ("counts", _Gpu((3,), i32, (2,))), ("positions", _Gpu((3,), i32)),
                      ("positions", _Gpu((3, 5), i32, (10, 2))), ("counts", _Gpu((3,), i32, device=1)), ("counts", 5)):
        with pytest.raises(ValueError):
            apply(**{name: bad})


class _Table(C.Structure):
    """A rotary handle of 16 dims on a device that there is not."""
    _fields_ = [("f", C.c_void_p), ("dims", C.c_int), ("interleaved", C.c_int), ("amplitude", C.c_float), ("device", C.c_int * 3)]


def test_rows_that_overlap_or_lie_askew_are_not_written(lib):
    r = C.byref(_Table(None, 16, 0, 1.0, (1 << 20, 0, 0)))
    x, out = 1 << 20, 1 << 21

    def apply(batch, n, out_strides, x=x, out=out, x_strides=(640, 64)):
        return lib.ravel_rotary_apply(r, batch, n, 2, 32, 1, x, *x_strides, out, *out_strides, None, None, None, None)

    # (a status of 1 is a refusal; what is not refused ends at the device)
    for batch, n, strides in ((3, 5, (640, 63)), (3, 5, (0, 64)), (3, 5, (319, 64)), (3, 5, (64, 191)), (3, 5, (64, 64)), (3, 1, (63, 0)),
                              (1, 5, (0, 0)), (2, 1 << 30, (1 << 62, 1 << 60))):
        assert apply(batch, n, strides) == 1 and b"overlap" in lib.ravel_decode_last_error(), strides
    assert apply(3, 5, (0, 64), out=x, x_strides=(0, 64)) == 1   # in place, robots that share their rows
    for batch, n, strides in ((3, 5, (320, 64)), (3, 5, (64, 192)), (3, 1, (64, 0)), (1, 5, (0, 64)), (1, 1, (0, 0)), (2, 2, (1 << 60, 1 << 61)), (2, 1 << 30, (1 << 40, 1 << 62))):
        apply(batch, n, strides)
        assert b"overlap" not in lib.ravel_decode_last_error(), strides
    assert apply(1, 1, (0, 0), x=x + 1) == 1 and b"unaligned" in lib.ravel_decode_last_error()
    assert apply(1, 1, (0, 0), out=out + 1) == 1 and b"unaligned" in lib.ravel_decode_last_error()
    p = C.c_void_p(256)
    assert lib.ravel_draw_tokens(C.c_void_p(258), 1, 8, 8, 0, p, None, None, None, None, p, None, None) == 1
    assert lib.ravel_w4_quantize(C.c_void_p(257), 8, 8, 8, 1, 32, p, p, p, None) == 1


def test_sizes_beyond_an_int_are_refused_not_cut_off(lib):
    import paper_2609_34170_gb300 as pkg
    b16, f32 = torch.bfloat16, torch.float32
    w = C.c_void_p()
    w.w4 = (256, 70, 32, 0)
    far = (1 << 32) + 72
    for x, out in ((_Gpu((4, 70), b16, (far, 1)), _Gpu((4, 256), b16)), (_Gpu((4, 70), b16), _Gpu((4, 256), b16, (far, 1))),
                   (_Gpu(((1 << 32) + 4, 70), b16), _Gpu(((1 << 32) + 4, 256), b16))):
        with pytest.raises(ValueError, match="2\\^31"):
            pkg.ravel_w4_gemm(w, x, 0, out, None, stream=0)
    with pytest.raises(ValueError, match="2\\^31"):
        pkg.ravel_draw_tokens(_Gpu((1, (1 << 32) + 4), f32), _Gpu((1,), f32), None, None, None, None, _Gpu((1,), torch.int32), stream=0)
    x = _Gpu((1, (1 << 32) + 4, 1, 16), b16)
    with pytest.raises(ValueError, match="2\\^31"):
        pkg.ravel_rotary_apply(_rotary_handle(), x, x, stream=0)
    from paper_2609_34170_gb300.decode import quantize4
    for bad in ((torch.zeros(4, 64), 32), (_Gpu((4, 64), f32), 48), (_Gpu((4, 64), f32), 0), (_Gpu((4,), f32), 32)):
        with pytest.raises(ValueError):
            quantize4(*bad)


def test_append_rotary_refuses_tensors_that_do_not_fit(lib):
    import paper_2609_34170_gb300 as pkg
    from paper_2609_34170_gb300 import _binding as B
    b16, i32 = torch.bfloat16, torch.int32
    c = C.c_void_p()
    c.arguments = B.CacheArguments(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=B.RAVEL_BF16, device=0)
    k, q, ints, pos = _Gpu((3, 5, 2, 64), b16), _Gpu((3, 5, 4, 64), b16), _Gpu((3,), i32), _Gpu((3, 5), i32)

    def append(r=_rotary_handle(), q=q, q_out=q, k=k, v=k, starts=ints, positions=pos, counts=ints):
        pkg.ravel_cache_append_rotary(c, 0, r, q, q_out, k, v, starts, positions, counts, stream=0)

    for good in (dict(), dict(q=None, q_out=None), dict(positions=None)):
        with pytest.raises(B.RavelError):
            append(**good)
    for bad in (dict(r=C.c_void_p()), dict(q=None), dict(q_out=None), dict(q=_Gpu((3, 4, 4, 64), b16)), dict(q_out=_Gpu((2, 5, 4, 64), b16)),
                dict(k=_Gpu((3, 5, 1, 64), b16)), dict(v=_Gpu((3, 4, 2, 64), b16)), dict(v=_Gpu((3, 5, 2, 64), torch.float32)),
                dict(positions=_Gpu((3, 4), i32)), dict(starts=_Gpu((2,), i32)), dict(counts=_Gpu((3,), torch.float32))):
        with pytest.raises(ValueError):
            append(**bad)


def test_products_refuse_tensors_that_do_not_fit(lib):
    import paper_2609_34170_gb300 as pkg
    from paper_2609_34170_gb300 import _binding as B
    b16, f32, u8 = torch.bfloat16, torch.float32, torch.uint8
    w = C.c_void_p()
    w.w4 = (256, 70, 32, 0)
    x, out = _Gpu((4, 70), b16, (72, 1)), _Gpu((4, 256), b16)

    def gemm(w=w, x=x, epi=0, out=out, bias=None):
        pkg.ravel_w4_gemm(w, x, epi, out, bias, stream=0)

    for good in (dict(), dict(epi=3, out=_Gpu((4, 128), b16)), dict(epi=2, out=_Gpu((4, 256), f32, (300, 1))), dict(bias=_Gpu((256,), f32))):
        with pytest.raises(B.RavelError):
            gemm(**good)
    for bad in (dict(w=C.c_void_p()), dict(x=_Gpu((4, 70), f32)), dict(x=_Gpu((4, 71), b16)), dict(x=_Gpu((4, 70), b16, (69, 1))),
                dict(x=_Gpu((4, 70), b16, (1, 4))), dict(x=_Gpu((4, 70), b16, device=1)), dict(out=_Gpu((3, 256), b16)),
                dict(out=_Gpu((4, 128), b16)), dict(out=_Gpu((4, 256), torch.float16)), dict(epi=3), dict(bias=_Gpu((128,), f32)),
                dict(bias=_Gpu((256,), b16))):
        with pytest.raises(ValueError):
            gemm(**bad)

    def load(codes=_Gpu((256, 35), u8), scales=_Gpu((256, 3), b16), zeros=_Gpu((256, 3), u8)):
        pkg.ravel_w4_load(w, codes, scales, zeros, stream=0)

    with pytest.raises(B.RavelError):
        load()
    for bad in (dict(codes=_Gpu((256, 70), u8)), dict(codes=_Gpu((256, 35), torch.int8)), dict(scales=_Gpu((256, 3), f32)),
                dict(scales=_Gpu((256, 2), b16)), dict(zeros=_Gpu((256, 3), u8, (6, 2)))):
        with pytest.raises(ValueError):
            load(**bad)


def test_draws_refuse_tensors_that_do_not_fit(lib):
    import paper_2609_34170_gb300 as pkg
    f32, i32 = torch.float32, torch.int32
    good = dict(logits=_Gpu((3, 50), f32), u=_Gpu((3,), f32), temperature=None, top_k=None, top_p=None, min_p=None, tokens=_Gpu((3,), i32),
                log_probs=_Gpu((3,), f32))
    for bad in (dict(logits=torch.zeros(3, 50)), dict(logits=_Gpu((3, 50), torch.float16)), dict(logits=_Gpu((150,), f32)),
                dict(logits=_Gpu((3, 50), f32, (1, 3))), dict(logits=_Gpu((3, 50), f32, (49, 1))), dict(u=None), dict(tokens=None),
                dict(u=_Gpu((2,), f32)), dict(temperature=0.7), dict(top_k=_Gpu((3,), f32)), dict(top_p=_Gpu((3,), i32)),
                dict(min_p=_Gpu((3, 1), f32)), dict(tokens=_Gpu((3,), torch.int64)), dict(log_probs=_Gpu((3,), torch.bfloat16))):
        with pytest.raises(ValueError):
            pkg.ravel_draw_tokens(**{**good, **bad}, stream=0)


def test_kernels_that_overlap_their_predecessors_read_nothing_as_constant():
    """Launches start before the ones before them end, which may write what they read: no load
    may take the read-only path.  (Weights and the rotary table, which nothing writes
    while they are used, are the exception.)"""
    import os

    from paper_2609_34170_gb300.build import CSRC
    for name in ("rotary.cu", "rotary.cuh", "w4.cu", "w4.cuh", "w4_tc.cu", "draw.cu"):
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        for word in ("__ldg(", "__ldcg(", "__ldcs(", "__ldca(", "ld.global.nc", "__restrict__"):
            assert word not in text, (name, word)


def test_waits_of_the_tensor_core_kernel_are_bounded():
    """Every wait goes through the helper that tries and then looks at the clock."""
    import os
    import re

    from paper_2609_34170_gb300.build import CSRC
    with open(os.path.join(CSRC, "w4_tc.cu")) as f:
        text = f.read()
    helper = text[text.index("bool wait_for("):text.index("template <int NTOK, int GS>\n__global__")]
    rest = text.replace(helper, "")
    assert "mbar_wait_warp" in helper and "wait_for(" in rest
    assert not re.search(r"mbar_(try_|test_)?wait", rest) and "while (!" not in rest and "bar.sync" not in rest
