"""The 8-bit context cache without a GPU: the fp64 reference against torch's
e4m3, its invariants, and what the library refuses before touching a device."""
import ctypes as C

import numpy as np
import pytest

from oracle import cache as ref

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lib():
    from paper_2609_34170_gb300 import build, load
    build.build()
    return load()


def test_reference_rounds_as_e4m3():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    codes = codes[np.isfinite(codes)]
    np.testing.assert_array_equal(ref.e4m3(codes), codes)
    x = np.random.default_rng(0).uniform(-448, 448, 20000) * 2.0 ** np.random.default_rng(1).integers(-18, 1, 20000)
    x = np.concatenate([x.astype(np.float32), (codes[:-1] + codes[1:]) / 2]).astype(np.float32)   # and ties
    np.testing.assert_array_equal(ref.e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


def test_reference_exponent_is_the_smallest_that_fits():
    for top in [448.0, np.nextafter(448.0, 500), 1.75, 1.7500001, 1e-30, 3e38, 2.0 ** -92 * 1.75]:
        e = ref.exponent(top)
        assert top <= 448 * 2.0 ** e and (e == ref.E_MIN or top > 448 * 2.0 ** (e - 1))
    assert ref.exponent(0.0) == ref.exponent(1e-40) == ref.E_MIN


def test_reference_append_in_pieces_holds_the_same_where_exponents_rise():
    """Values stored token by token differ from those stored at once by no more
    than a second rounding: half a step of the final grid's smallest."""
    rng = np.random.default_rng(2)
    k = rng.standard_normal((1, 16, 1, 8)) * 2.0 ** np.arange(16)[None, :, None, None]
    one, many = ref.Held(1, 1, 16, 8), ref.Held(1, 1, 16, 8)
    one.append(k, k, [0], [16])
    for i in range(16):
        many.append(k[:, i:i + 1], k[:, i:i + 1], [i], [1])
    assert one.ke[0, 0, 0] == many.ke[0, 0, 0]
    step = 2.0 ** (one.ke[0, 0, 0] - 9)
    rel = np.abs(one.k - k.transpose(0, 2, 1, 3)).max()
    assert np.abs(one.k - many.k).max() <= np.maximum(step, rel)


def test_create_refuses_bad_shapes_without_a_gpu(lib):
    from paper_2609_34170_gb300 import RavelError, ravel_cache_create
    good = dict(layers=1, n_q_heads=4, n_kv_heads=2, head_dim=64, max_tokens=32, max_batch=1, max_queries=1)
    for bad in (dict(layers=0), dict(n_q_heads=3), dict(head_dim=12), dict(head_dim=264), dict(max_tokens=0),
                dict(max_batch=0), dict(max_queries=0), dict(dtype=2), dict(max_batch=65536), dict(n_kv_heads=0),
                dict(max_tokens=(1 << 30) + 1), dict(max_queries=1 << 30)):
        with pytest.raises(RavelError) as ei:
            ravel_cache_create(**{**good, **bad})
        assert ei.value.status == 2
    with pytest.raises(ValueError):
        from paper_2609_34170_gb300 import ContextCache
        ContextCache(layers=1, n_q_heads=1, n_kv_heads=1, head_dim=64, max_tokens=16, dtype="fp16")


def test_null_arguments_are_refused(lib):
    assert lib.ravel_cache_create(None, 0, None) == 1
    assert lib.ravel_cache_append(None, 0, 1, 1, None, None, 0, 0, None, None, None) == 1
    assert lib.ravel_cache_attend(None, 0, 1, 1, None, 0, 0, None, 0, 0, None, None, 0, 1, 0, 0, 0.0, None, 0, 0, None) == 1
    assert lib.ravel_cache_evict(None, 0, None, 0, 1, None, None, 0, 1, 0, 0, None, None, None, None) == 1
    assert lib.ravel_cache_read(None, 0, 1, 1, None, None, None, None, None) == 1
    assert lib.ravel_cache_reset(None) == 1
    assert lib.ravel_cache_last_error(None) == b""
    lib.ravel_cache_destroy(None)


def test_binding_refuses_tensors_of_the_wrong_kind(lib):
    from paper_2609_34170_gb300 import ravel_cache_append, ravel_cache_attend
    handle = C.c_void_p()
    k = torch.zeros((1, 2, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):   # not on a GPU
        ravel_cache_append(handle, 0, k, k)
    with pytest.raises(ValueError):
        ravel_cache_attend(handle, 0, k, k, None, None, 2)


class _Gpu:
    """Stands in for a CUDA tensor: all that the calls look at, none of the memory."""
    is_cuda = True

    def __init__(self, shape, dtype, stride=None, device=0):
        self.shape, self.dtype, self.device, self._device = torch.Size(shape), dtype, torch.device("cuda", device), device
        dense = [1]
        for n in reversed(shape[1:]):
            dense.insert(0, dense[0] * n)
        self._stride = tuple(stride or dense)
        self._dense = self._stride == tuple(dense)

    def stride(self):
        return self._stride

    def get_device(self):
        return self._device

    def is_contiguous(self):
        return self._dense

    def data_ptr(self):
        return 256


def test_calls_on_a_handle_check_their_tensors_against_the_cache(lib):
    """What does not fit the cache would be read or written past its end: it is
    refused before the library is called (whose refusal of the null handle is a
    RavelError)."""
    import paper_2609_34170_gb300 as pkg
    from paper_2609_34170_gb300 import _binding as B
    c, to = C.c_void_p(), C.c_void_p()
    for h in (c, to):
        h.arguments = B.CacheArguments(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=B.RAVEL_BF16, device=0)
    b16, f32, i32, u32 = torch.bfloat16, torch.float32, torch.int32, torch.uint32
    k, q, ints = _Gpu((3, 5, 2, 64), b16), _Gpu((3, 5, 4, 64), b16), _Gpu((3,), i32)
    mass, held = _Gpu((3, 2, 40), f32), _Gpu((3, 2, 9, 64), b16)
    index, new_mass = _Gpu((3, 2, 8), i32), _Gpu((3, 2, 8), f32)

    def append(h=c, k=k, v=None, starts=None, counts=None):
        pkg.ravel_cache_append(h, 0, k, v or k, starts, counts, stream=0)

    def attend(h=c, q=q, out=None, lengths=ints, counts=None, mass=None):
        pkg.ravel_cache_attend(h, 0, q, out or q, lengths, counts, 40, mass=mass, stream=0)

    def evict(h=c, to=to, lengths=ints, mass=mass, new_lengths=ints, index=index, new_mass=new_mass):
        pkg.ravel_cache_evict(h, 0, to, 0, lengths, mass, 8, 1, 1, new_lengths, index, new_mass, stream=0)

    def read(h=c, k=held, v=None, firsts=None, lengths=None):
        pkg.ravel_cache_read(h, 0, k, v or k, firsts, lengths, stream=0)

    for call in (append, attend, evict, read):   # what fits goes to the library
        with pytest.raises(B.RavelError) as ei:
            call()
        assert ei.value.status == 1
        with pytest.raises(ValueError):
            call(h=C.c_void_p())
    wrong_ints = [_Gpu((2,), i32), _Gpu((3,), u32), _Gpu((3,), f32), _Gpu((3,), i32, (2,)), _Gpu((3,), i32, device=1)]
    for bad in (_Gpu((3, 5, 2, 64), f32), _Gpu((3, 5, 1, 64), b16), _Gpu((3, 5, 2, 32), b16), _Gpu((3, 5, 128), b16),
                _Gpu((3, 5, 2, 64), b16, device=1), _Gpu((3, 5, 2, 64), b16, (640, 64, 320, 1))):
        for args in (dict(k=bad), dict(v=bad)):
            with pytest.raises(ValueError):
                append(**args)
    for bad in (_Gpu((3, 5, 4, 64), f32), _Gpu((3, 5, 3, 64), b16), _Gpu((3, 5, 4, 72), b16), _Gpu((3, 5, 4, 64), b16, device=1)):
        for args in (dict(q=bad), dict(out=bad)):
            with pytest.raises(ValueError):
                attend(**args)
    for bad in (_Gpu((2, 2, 40), f32), _Gpu((3, 1, 40), f32), _Gpu((3, 2, 40), b16), _Gpu((6, 40), f32),
                _Gpu((3, 2, 40), f32, (160, 80, 2))):
        with pytest.raises(ValueError):
            attend(mass=bad)
        with pytest.raises(ValueError):
            evict(mass=bad)
    for bad in (_Gpu((3, 2, 7), i32), _Gpu((3, 1, 8), i32), _Gpu((3, 2, 8), f32), _Gpu((2, 2, 8), i32)):
        with pytest.raises(ValueError):
            evict(index=bad)
    for bad in (_Gpu((3, 2, 7), f32), _Gpu((3, 2, 8), i32)):
        with pytest.raises(ValueError):
            evict(new_mass=bad)
    for bad in (_Gpu((3, 2, 9, 64), f32), _Gpu((3, 1, 9, 64), b16), _Gpu((3, 2, 9, 32), b16), _Gpu((3, 2, 576), b16)):
        for args in (dict(k=bad), dict(v=bad)):
            with pytest.raises(ValueError):
                read(**args)
    for bad in wrong_ints:
        for call, names in ((append, ("starts", "counts")), (attend, ("lengths", "counts")), (evict, ("lengths", "new_lengths")),
                            (read, ("firsts", "lengths"))):
            for name in names:
                with pytest.raises(ValueError):
                    call(**{name: bad})


def test_kernels_that_overlap_their_predecessors_read_nothing_as_constant():
    """The cache's launches start before the ones before them end, which may write
    what they read: no load may take the read-only path or pass the wait in front
    of it (those of the read-only kind, restrict pointers, loads that the compiler
    takes for pure functions)."""
    import glob
    import os

    from paper_2609_34170_gb300.build import CSRC
    files = glob.glob(os.path.join(CSRC, "cache*.cu*"))
    assert len(files) >= 6
    for path in files:
        with open(path) as f:
            text = f.read()
        for word in ("__ldg(", "__ldcg(", "__ldcs(", "__ldca(", "ld.global.nc", "__restrict__"):
            assert word not in text, (os.path.basename(path), word)
        for line in text.splitlines():
            assert "ld.global" not in line or "asm volatile" in line, line


def test_create_refuses_positions_that_could_pass_32_bits(lib):
    """A CTA steps up to 2^14 tokens past the last one."""
    from paper_2609_34170_gb300 import RavelError, ravel_cache_create
    for batch, heads in ((1, 1), (2, 4)):
        most = (2 ** 31 - 2 ** 16) // (batch * heads) - 128
        for tokens in (most + 1, most + 2 ** 15 // (batch * heads), 2 ** 31 // (batch * heads) - 129):
            with pytest.raises(RavelError) as ei:
                ravel_cache_create(layers=1, n_q_heads=4, n_kv_heads=heads, head_dim=64, max_tokens=tokens, max_batch=batch,
                                   max_queries=1)
            assert ei.value.status == 2


def test_strides_of_a_single_robot_or_token_mean_nothing(lib):
    import paper_2609_34170_gb300 as pkg
    from paper_2609_34170_gb300 import _binding as B
    c = C.c_void_p()
    c.arguments = B.CacheArguments(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=B.RAVEL_BF16, device=0)

    def append(shape, k_stride, v_stride):
        pkg.ravel_cache_append(c, 0, _Gpu(shape, torch.bfloat16, k_stride), _Gpu(shape, torch.bfloat16, v_stride), stream=0)

    for shape, k, v in (((1, 1, 2, 64), (128, 128, 64, 1), (512, 512, 64, 1)), ((1, 5, 2, 64), (640, 512, 64, 1), (9999, 512, 64, 1)),
                        ((3, 1, 2, 64), (512, 128, 64, 1), (512, 512, 64, 1))):
        with pytest.raises(B.RavelError):     # (by the library: the handle is null)
            append(shape, k, v)
    for shape, k, v in (((1, 5, 2, 64), (640, 128, 64, 1), (640, 512, 64, 1)), ((3, 1, 2, 64), (128, 128, 64, 1), (512, 128, 64, 1))):
        with pytest.raises(ValueError):
            append(shape, k, v)
    assert c.arguments.rows(_Gpu((1, 1, 2, 64), torch.bfloat16, (7, 3, 64, 1)), 2, "k") == (0, 0)


def test_two_pieces_hold_what_the_prompts_kernels_claim():
    """y = e4m3(y) + e5m2(rest) for bf16 values of a row whose largest lies in [2^7, 2^8): exact from
    2^-6 on, off by at most 2^-14 below."""
    bits = torch.arange(1 << 15, dtype=torch.int32)
    y = bits.to(torch.int16).view(torch.bfloat16).double()
    y = y[(y < 2.0 ** 8) & (y > 2.0 ** -60)]
    half = y.to(torch.float16)        # (a subnormal's rounding, below 2^-14)
    hi = half.to(torch.float8_e4m3fn)
    lo = (half - hi.half()).to(torch.float8_e5m2)
    off = (y - hi.double() - lo.double()).abs()
    assert (off[y >= 2.0 ** -6] == 0).all() and off.max() <= 2.0 ** -14
