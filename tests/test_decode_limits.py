"""Rotary positions, 4-bit products and drawing tokens without a GPU: settings at the ends of what the calls can hold."""
import ctypes as C
import math

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lib():
    from paper_2609_34170_gb300 import build, load
    build.build()
    return load()


@pytest.mark.parametrize("bad", [dict(factor=1e-310), dict(base=1e-320, dims=256), dict(base=5e-324, factor=1e-200), dict(amplitude=1e39),
                                 dict(amplitude=-3.5e38), dict(base=1e-300, factor=1e-60, original_length=1e-3, low=0.0, high=1e300)])
def test_rotary_refuses_settings_whose_table_is_not_finite(lib, bad):
    """Each is finite; the frequencies that they make, or the amplitude in fp32, are not."""
    from paper_2609_34170_gb300 import RavelError, ravel_rotary_create
    with pytest.raises(RavelError) as ei:
        ravel_rotary_create(**{**dict(dims=16), **bad})
    assert ei.value.status == 1 and "finite" in str(ei.value)


def _wide(of: int) -> int:
    """What an int of 32 bits makes `of` from."""
    return of + (1 << 32)


def test_settings_beyond_an_int_are_refused_not_cut_off(lib):
    """ctypes passes the low 32 bits of a Python int: a matrix of other sizes than the handle's, a group of 32 for scales
    of one group a row (read past their end)."""
    import paper_2609_34170_gb300 as pkg
    from tests.test_decode_host import _Gpu
    for args in ((_wide(96), 64, 32), (96, _wide(64), 32), (96, 64, _wide(32)), (96, 64, 32, _wide(0)), (96, 64, 32 - (1 << 32))):
        with pytest.raises(ValueError, match="2\\^31"):
            pkg.ravel_w4_create(*args)
    with pytest.raises(ValueError, match="2\\^31"):
        pkg.ravel_rotary_create(_wide(16))
    with pytest.raises(ValueError, match="2\\^31"):
        pkg.ravel_rotary_create(16, device=_wide(0))
    f32, b16, u8 = torch.float32, torch.bfloat16, torch.uint8
    with pytest.raises(ValueError, match="2\\^31"):
        pkg.ravel_w4_quantize(_Gpu((4, 64), f32), _wide(32), _Gpu((4, 32), u8), _Gpu((4, 1), b16), _Gpu((4, 1), u8), stream=0)
    w = C.c_void_p()
    w.w4 = (256, 70, 32, 0)
    with pytest.raises(ValueError, match="epilogue"):
        pkg.ravel_w4_gemm(w, _Gpu((4, 70), b16), _wide(3), _Gpu((4, 256), b16), None, stream=0)


def test_append_rotary_refuses_sizes_beyond_an_int(lib):
    """(k of one robot seen 2^32 + 1 times would be stored once)"""
    import paper_2609_34170_gb300 as pkg
    from paper_2609_34170_gb300 import _binding as B
    from tests.test_decode_host import _Gpu, _rotary_handle
    c = C.c_void_p()
    c.arguments = B.CacheArguments(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=B.RAVEL_BF16, device=0)
    cache = pkg.ContextCache.__new__(pkg.ContextCache)
    cache.handle, cache._lib, cache._rows, cache._ints, cache._dense = c, lib, c.arguments.rows, c.arguments.ints, c.arguments.dense
    cache.n_q_heads, cache.n_kv_heads, cache._stream = 4, 2, lambda stream: 0
    rotary = pkg.Rotary.__new__(pkg.Rotary)
    rotary.handle = _rotary_handle()
    for layer, shape, stride in ((0, (_wide(1), 3, 2, 64), (0, 128, 64, 1)), (0, (3, _wide(1), 2, 64), (128, 0, 64, 1)),
                                 (_wide(0), (3, 5, 2, 64), None)):
        k = _Gpu(shape, torch.bfloat16, stride)
        with pytest.raises(ValueError, match="2\\^31"):
            pkg.ravel_cache_append_rotary(c, layer, rotary.handle, None, None, k, k, stream=0)
        with pytest.raises(ValueError, match="2\\^31"):
            cache.append_rotary(layer, rotary, None, k, k)
    rotary.handle = cache.handle = None   # (nothing to close)


def test_types_are_looked_up_before_another_thread_may_use_them():
    """Two threads' first calls: whoever finds the look-up done finds all of it.  (Looked at after each instruction.)"""
    import sys

    from paper_2609_34170_gb300 import _binding as B

    class Fresh(B._Types):
        bf16 = f32 = i32 = u8 = get_device = None

    seen = []

    def watch(frame, event, arg):
        if frame.f_code.co_name != "look_up":
            return None
        frame.f_trace_opcodes = True
        if Fresh.bf16 is not None:
            seen.append(None not in (Fresh.f32, Fresh.i32, Fresh.u8, Fresh.get_device))
        return watch

    sys.settrace(watch)
    try:
        Fresh.look_up()
    finally:
        sys.settrace(None)
    assert seen and all(seen) and Fresh.bf16 is torch.bfloat16


class _Matrix(C.Structure):
    """A handle of a 4-bit matrix as far as its error word's mirror, on a device that there is not."""
    _fields_ = [("codes", C.c_void_p), ("sz", C.c_void_p), ("sizes", C.c_int * 6), ("device", C.c_int * 2), ("err", C.c_void_p),
                ("err_host", C.POINTER(C.c_int))]


def test_an_error_of_earlier_work_is_reported_before_a_device_is_touched(lib):
    word = C.c_int(0)
    w = C.byref(_Matrix(None, None, (96, 64, 32, 6, 1, 2), (1 << 20, 0), None, C.pointer(word)))
    for bits, status in ((1 << 1, 8), (1 << 2, 7), (3 << 1, 8)):   # a wait that ran out; any other
        word.value = bits
        assert lib.ravel_w4_gemm(w, 1 << 20, 3, 64, 0, 1 << 21, 96, 0, None, None) == status
        assert b"error word" in lib.ravel_decode_last_error()
        assert lib.ravel_w4_gemm(w, 1 << 20, 0, 64, 0, 1 << 21, 96, 0, None, None) == 0   # nothing to do
    word.value = 0
    lib.ravel_w4_gemm(w, 1 << 20, 3, 64, 0, 1 << 21, 96, 0, None, None)   # (ends at the device)
    assert b"error word" not in lib.ravel_decode_last_error()
