"""Rotary positions, 4-bit products and drawing tokens at the largest sizes and strides: counts of rows, robots and
weights that the headers name, and addresses more than 2^31 values apart."""
import math

import numpy as np
import pytest

from oracle import decode as ref
from tests.test_gpu_decode import _draws, _ints, _lib, _np, _rand, _turn_close  # noqa: F401
from tests.test_gpu_decode_tc import kernel  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _matrix(n, k, group, seed):
    from paper_2609_34170_gb300 import Weights4
    g = torch.Generator("cuda").manual_seed(seed)
    groups = -(-k // group)
    codes = torch.randint(0, 256, (n, (k + 1) // 2), generator=g, dtype=torch.uint8, device="cuda")
    scales = ((torch.rand((n, groups), generator=g, device="cuda") + 0.1) / math.sqrt(k)).to(torch.bfloat16)
    zeros = torch.randint(0, 16, (n, groups), generator=g, dtype=torch.uint8, device="cuda")
    w = Weights4(n, k, group)
    w.load(codes, scales, zeros)
    return w, codes, scales, zeros


def _values(codes, scales, zeros, k, group):
    """[N, K] in 64 bits, on the GPU."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(1)[:, :k].double()
    at = torch.arange(k, device="cuda") // group
    return (c - zeros.double()[:, at]) * scales.double()[:, at]


def _close(got, x, held):
    """test_gpu_decode.py's tolerance, fp32 out."""
    x = x.double()
    y = x @ held.t()
    tol = (2.0 ** -19 + (held.shape[1] / 32 + 18) * 2.0 ** -24) * (x.abs() @ held.abs().t()) + 2.0 ** -22 * y.abs()
    assert ((got.double() - y).abs() <= tol).all()


def test_rows_far_apart_are_turned_and_drawn_from():
    """Five rows over 9 GB."""
    far = 1150000008   # (a multiple of 8; twice and four times it pass 2^31 and 2^32)
    flat = torch.empty((4 * far + 5000,), dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((5, 3, 2, 64), (far, 128, 64, 1))
    x.copy_(_rand((5, 3, 2, 64), 0, "bf16"))
    from paper_2609_34170_gb300 import ContextCache, Rotary
    r, want = Rotary(64), x.contiguous()
    turned = r.apply(want, starts=_ints([7] * 5))
    assert torch.equal(r.apply(x, starts=_ints([7] * 5)), turned)
    cache, plain = ContextCache(1, 2, 2, 64, 16, 5), ContextCache(1, 2, 2, 64, 16, 5)
    cache.append_rotary(0, r, x, x, x, _ints([7] * 5), q_out=x)   # in place, robots far apart
    assert torch.equal(x, turned)
    x.copy_(want)
    cache.append_rotary(0, r, None, x, x, _ints([7] * 5))
    plain.append_rotary(0, r, None, want, want, _ints([7] * 5))
    assert all(torch.equal(a, b) for a, b in zip(cache.read(0, 5, 12), plain.read(0, 5, 12)))
    y = flat.as_strided((5, 4099), (far, 1))
    y.copy_(_rand((5, 4099), 1, "bf16", 3.0))
    _draws(y, [0.1, 0.3, 0.5, 0.7, 0.9], k=[50] * 5, p=[0.9] * 5)
    _draws(y, [0.1, 0.3, 0.5, 0.7, 0.9], p=[0.9] * 5)


def test_products_of_rows_far_apart(kernel):
    far = 550000000
    w, codes, scales, zeros = _matrix(300, 520, 64, 0)
    held = _values(codes, scales, zeros, 520, 64)
    x = torch.empty((11 * far + 600,), dtype=torch.bfloat16, device="cuda").as_strided((12, 520), (far, 1))
    x.copy_(_rand((12, 520), 1, "bf16"))
    _close(w.product(x, dtype=torch.float32), x, held)
    _close(w.product(x[:5], dtype=torch.float32), x[:5], held)
    near = x.contiguous()
    del x
    out = torch.empty((11 * far + 400,), device="cuda").as_strided((12, 300), (far, 1))
    for m in (12, 5):
        out.zero_()
        _close(w.product(near[:m], out=out[:m]), near[:m], held)
        _close(w.product(near[:m], out=out[:m], epi="add") / 2, near[:m], held)   # (twice: half of it is exact)


def test_products_of_half_a_million_rows(kernel):
    w, codes, scales, zeros = _matrix(33, 72, 32, 1)
    held = _values(codes, scales, zeros, 72, 32)
    x = _rand((1 << 19, 72), 2, "bf16")
    _close(w.product(x, dtype=torch.float32), x, held)
    x = x[:100003]
    _close(w.product(x, dtype=torch.float32), x, held)


@pytest.mark.parametrize("n,k,group", [(1 << 24, 40, 32), (17, 1 << 24, 128), (33, (1 << 24) - 3, 32)])
def test_products_of_the_longest_and_the_widest_matrices(kernel, n, k, group):
    w, codes, scales, zeros = _matrix(n, k, group, 2)
    for m in (1, 12, 40):
        x = _rand((m, -(-k // 8) * 8), m, "bf16")[:, :k]
        got = w.product(x, dtype=torch.float32)
        for at in range(0, n, 1 << 21) if n > 1000 else range(n):
            part = slice(at, at + (4099 if n > 1000 else 1))
            _close(got[:, part], x, _values(codes[part], scales[part], zeros[part], k, group))
        part = slice(max(n - 200, 0), n) if n > 1000 else slice(n - 1, n)
        _close(got[:, part], x, _values(codes[part], scales[part], zeros[part], k, group))


def test_products_of_a_matrix_of_more_than_four_gigabytes(kernel):
    n, k = 140001, 65600
    w, codes, scales, zeros = _matrix(n, k, 64, 3)
    parts = [slice(0, 300), slice(65400, 65700), slice(131000, 131200), slice(n - 260, n)]   # (2^32 bytes of codes end at row 130945)
    for m in (1, 12, 40):
        x = _rand((m, k), m, "bf16")
        got = w.product(x, dtype=torch.float32)
        for part in parts:
            _close(got[:, part], x, _values(codes[part], scales[part], zeros[part], k, 64))


def test_as_many_robots_as_a_call_takes():
    from paper_2609_34170_gb300 import RavelError, Rotary, draw_tokens
    many = 65535
    x = _rand((many, 2, 1, 16), 0, "bf16")
    starts = np.arange(many) * 3
    got = Rotary(16).apply(x, starts=_ints(starts))
    _turn_close(_np(got), _np(x), starts[:, None] + np.arange(2), ref.frequencies(16), 16, False, "bf16")
    x, u = _rand((many, 9), 1, "fp32", 2.0), np.random.default_rng(2).random(many, dtype=np.float32)
    _draws(x, u, p=[0.8] * many)
    for call in (lambda: Rotary(16).apply(torch.zeros((many + 1, 1, 1, 16), device="cuda")),
                 lambda: draw_tokens(torch.zeros((many + 1, 3), device="cuda"), torch.zeros((many + 1,), device="cuda"))):
        with pytest.raises(RavelError) as ei:
            call()
        assert ei.value.status == 2


def test_turns_millions_of_tokens_and_tens_of_thousands_of_heads():
    from paper_2609_34170_gb300 import Rotary
    for shape, dims in (((1, 5000011, 1, 4), 4), ((2, 3, 65535, 8), 6), ((1, 700000, 3, 256), 256)):
        x = _rand(shape, 3, "bf16")
        got = Rotary(dims).apply(x, starts=_ints([5] * shape[0]))
        for at in (0, shape[1] // 2, shape[1] - 3):
            here = x[:, at:at + 3]
            assert torch.equal(got[:, at:at + 3], Rotary(dims).apply(here, starts=_ints([5 + at] * shape[0])))
        at = shape[1] - 3
        tail = slice(-5, None)
        _turn_close(_np(got[:, at:, tail]), _np(x[:, at:, tail]), 5 + np.arange(at, shape[1])[None] + np.zeros((shape[0], 1), int),
                    ref.frequencies(dims), dims, False, "bf16")
