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
