"""4-bit products of more than 8 rows on either kernel (tcgen05, and tiles of 16 rows) whatever the rule between them
says of their sizes: small and ragged ones, every epilogue and group, 1, 2 and 4 CTAs to a unit, full rounds before a
shared one, values behind K, captures and streams.

Tolerance: that of test_gpu_decode.py, whose parts hold here: a chain of at most eight MMAs of 16 ks from zero, 2^-19 of
the group's sum of magnitudes; then a sum over the groups, K / 32 at most, and over at most 4 CTAs, and the bias, 2^-24
each: (2^-19 + (K / 32 + 4) 2^-24) sum |x w|, below the (2^-19 + (K / 32 + 18) 2^-24) that is allowed."""
import ctypes as C
import os
import subprocess
import sys

import numpy as np
import pytest

from tests.test_gpu_decode import _held, _lib, _np, _product_close, _rand  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TILES, TC = 1, 2


def _plan(n, k, group, m):
    """Kernel, tokens of a unit, CTAs, CTAs to a unit, full rounds."""
    from paper_2609_34170_gb300 import load
    out = (C.c_int * 5)()
    load().ravel_debug_w4_plan(n, k, group, m, 1, torch.cuda.get_device_properties(0).multi_processor_count, out)
    return tuple(out)


@pytest.fixture(params=[TILES, TC], ids=["tiles", "tcgen05"])
def kernel(request):
    from paper_2609_34170_gb300 import load
    load().ravel_debug_w4(request.param)
    yield request.param
    load().ravel_debug_w4(-1)


def _tokens(m, k, seed):
    """Aligned rows of k values with NaN behind them."""
    x = torch.full((m, -(-k // 8) * 8 + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    x[:, :k] = _rand((m, k), seed, "bf16")
    return x[:, :k]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,k", [(1, 1), (16, 64), (31, 40), (33, 130), (77, 1003), (640, 1024), (128, 4096), (1000, 520), (129, 8200)])
def test_products_of_all_sizes(kernel, n, k, group):
    w, held = _held(n, k, group, n + k)
    bias = _rand((n,), 3)
    for m in (9, 16, 17, 31, 32, 33, 64, 65, 130):
        assert _plan(n, k, group, m)[0] == kernel
        x = _tokens(m, k, m)
        for epi, dtype, b in (("store", "bf16", None), ("silu", "fp32", bias), ("add", "fp32", None), ("store", "fp32", bias)):
            before = _rand((m, n), m + 1)
            got = w.product(x, out=before.clone() if epi == "add" else None, epi=epi, bias=b,
                            dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
            _product_close(_np(got), _np(x), held, epi, dtype, None if b is None else _np(b), _np(before))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,k", [(128, 64), (384, 333), (2560, 1500)])
def test_geglu_products(kernel, n, k, group):
    w, held = _held(n, k, group, n)
    bias = _rand((n,), 4)
    for m in (9, 32, 50, 72):
        x = _tokens(m, k, m)
        _product_close(_np(w.product(x, epi="geglu")), _np(x), held, "geglu", "bf16")
        _product_close(_np(w.product(x, epi="geglu", bias=bias)), _np(x), held, "geglu", "bf16", _np(bias))


@pytest.mark.parametrize("kernel", [TC], indirect=True)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("tokens,m", [(32, 12), (32, 29), (64, 40), (64, 64)])
@pytest.mark.parametrize("n,k,ranks,rounds", [(256, 260, 1, 0), (256, 600, 2, 0), (384, 1100, 4, 0), (20480, 260, 1, 1), (20480, 600, 2, 1)])
def test_products_of_every_plan(kernel, n, k, ranks, rounds, tokens, m, group):
    """How many CTAs share a unit's ks, with and without full rounds before."""
    assert _plan(n, k, group, m)[:2] + _plan(n, k, group, m)[3:] == (TC, tokens, ranks, rounds)
    w, held = _held(n, k, group, k)
    x, bias, before = _tokens(m, k, 1), _rand((n,), 4), _rand((m, n), 2)
    _product_close(_np(w.product(x, epi="geglu", bias=bias)), _np(x), held, "geglu", "bf16", _np(bias))
    _product_close(_np(w.product(x, epi="silu", dtype=torch.float32)), _np(x), held, "silu", "fp32")
    _product_close(_np(w.product(x)), _np(x), held, "store", "bf16")
    _product_close(_np(w.product(x, out=before.clone(), epi="add", bias=bias)), _np(x), held, "add", "fp32", _np(bias), _np(before))


@pytest.mark.parametrize("group", [32, 128])
def test_values_that_are_not_finite_stay_in_their_rows(kernel, group):
    w, held = _held(40, 100, group)
    x = _tokens(20, 100, 6)
    x[2, 50] = float("inf")
    x[13, 1] = float("nan")
    got = _np(w.product(x, dtype=torch.float32))
    rows = [i for i in range(20) if i not in (2, 13)]
    _product_close(got[rows], _np(x)[rows], held, "store", "fp32")
    assert not np.isfinite(got[2]).all() and np.isnan(got[13]).all()


def test_products_touch_nothing_else(kernel):
    """Rows of out that lie apart, and rows behind the last token."""
    for n, k, m in ((50, 104, 20), (20449, 300, 33)):
        w, held = _held(n, k, 64)
        x = _tokens(m, k, 5)
        out = torch.full((m + 40, n + 11), -5.0, device="cuda")
        w.product(x, out=out[:m, 3:n + 3])
        _product_close(_np(out[:m, 3:n + 3]), _np(x), held, "store", "fp32")
        assert (out[:, :3] == -5).all() and (out[:, n + 3:] == -5).all() and (out[m:] == -5).all()


def test_two_streams_and_two_graphs_share_weights(kernel):
    """Launches side by side: whole SMs each, clusters that wait for their own CTAs."""
    cases = []
    for n, k, m in ((20480, 600, 58), (384, 1100, 29)):
        w, held = _held(n, k, 128, n)
        xs = [_tokens(m, k, seed) for seed in (1, 2)]
        want = [w.product(x, dtype=torch.float32) for x in xs]
        for x, y in zip(xs, want):
            _product_close(_np(y), _np(x), held, "store", "fp32")
        cases.append((w, xs, want))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i in range(30):
        for j, s in enumerate(streams):
            w, xs, want = cases[(i + j) % 2]
            got.append((w.product(xs[j], dtype=torch.float32, stream=s), want[j]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in got)
    graphs, outs = [], []
    for j, s in enumerate(streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs.append([w.product(xs[j], dtype=torch.float32) for w, xs, _ in cases * 3])
        graphs.append(graph)
    for _ in range(5):
        for j, s in enumerate(streams):
            with torch.cuda.stream(s):
                graphs[j].replay()
    torch.cuda.synchronize()
    for j in range(2):
        assert all(torch.equal(a, want[j]) for a, (_, _, want) in zip(outs[j], cases * 3))


FIRST_CALLS = """
import sys; sys.path.insert(0, sys.argv[1])
import math, torch
from paper_2609_34170_gb300 import Weights4, load
load().ravel_debug_w4(int(sys.argv[2]))
g = torch.Generator("cuda").manual_seed(0)
made = []
for n, k, m in ((4200, 512, 40), (384, 1096, 20), (20480, 600, 58), (100, 64, 5)):
    w = Weights4(n, k, 64)
    codes = torch.randint(0, 256, (n, k // 2), generator=g, dtype=torch.uint8, device="cuda")
    zeros = torch.randint(0, 16, (n, -(-k // 64)), generator=g, dtype=torch.uint8, device="cuda")
    scales = (torch.rand(zeros.shape, generator=g, device="cuda") / math.sqrt(k)).to(torch.bfloat16)
    w.load(codes, scales, zeros)
    made.append((w, torch.randn((m, k), generator=g, device="cuda").to(torch.bfloat16)))
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = [w.product(x, dtype=torch.float32) for w, x in made]
graph.replay()
torch.cuda.synchronize()
for (w, x), y in zip(made, got):
    held = w.read(torch.float32).double().cpu()
    x = x.double().cpu()
    tol = (2.0 ** -19 + (held.shape[1] / 32 + 18) * 2.0 ** -24) * (x.abs() @ held.abs().t()) + 2.0 ** -22 * (x @ held.t()).abs()
    assert (held != 0).any() and ((y.double().cpu() - x @ held.t()).abs() <= tol).all()
    assert torch.equal(w.product(x.cuda().to(torch.bfloat16), dtype=torch.float32), y)
print("the same")
"""


@pytest.mark.parametrize("which", [-1, TILES, TC])
def test_first_calls_may_be_captured(which):
    """In a process of its own, where nothing has run before the capture."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", FIRST_CALLS, root, str(which)], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "the same" in done.stdout, done.stderr[-2000:]


@pytest.mark.parametrize("kernel", [TC], indirect=True)
@pytest.mark.parametrize("n,k,m,group", [(256, 260, 20, 128), (384, 1100, 40, 64), (20480, 600, 58, 32)])
def test_a_wait_that_runs_out_is_reported_until_a_reset(kernel, n, k, m, group):
    """Tokens that are not loaded: the roles' waits give up after a second, later products of the matrix (of any number of
    rows) are refused, others are not, and after a reset they are what they were."""
    from paper_2609_34170_gb300 import RavelError, load
    w, held = _held(n, k, group, n)
    other, _ = _held(256, 260, 128, 1)
    x, y = _tokens(m, k, 1), _tokens(20, 260, 2)
    want, untouched = w.product(x, dtype=torch.float32), other.product(y)
    _product_close(_np(want), _np(x), held, "store", "fp32")
    load().ravel_debug_w4_withhold(1)
    w.product(x, dtype=torch.float32)
    torch.cuda.synchronize()
    for rows in (x, x[:3]):
        with pytest.raises(RavelError) as ei:
            w.product(rows)
        assert ei.value.status == 8   # RAVEL_ETIMEOUT
    assert torch.equal(other.product(y), untouched)
    np.testing.assert_array_equal(_np(w.read(torch.float32)), held.astype(np.float32))
    w.reset()
    assert torch.equal(w.product(x, dtype=torch.float32), want)
