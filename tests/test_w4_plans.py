"""Which kernel takes a 4-bit product and what the tcgen05 kernel cuts it into (host code, no GPU)."""
import ctypes as C
import random

import pytest

pytest.importorskip("torch")

FEW, TILES, TC = 0, 1, 2
SMS = 152


@pytest.fixture(scope="module")
def lib():
    from paper_2609_34170_gb300 import build, load
    build.build()
    return load()


def _plan(lib, n, k, group, m, aligned=1):
    out = (C.c_int * 5)()
    lib.ravel_debug_w4_plan(n, k, group, m, aligned, SMS, out)
    return dict(zip(("kernel", "tokens", "grid", "ranks", "rounds"), out))


def _draws(count, seed):
    rng = random.Random(seed)
    for _ in range(count):
        yield int(2 ** rng.uniform(0, 17)), int(2 ** rng.uniform(0, 15)), rng.choice([32, 64, 128]), int(2 ** rng.uniform(0, 9))


def test_few_and_unaligned_rows_stay_off_tensor_memory(lib):
    for n, k, group, m in _draws(3000, 0):
        assert (_plan(lib, n, k, group, m)["kernel"] == FEW) == (m <= 8)
        assert _plan(lib, n, k, group, m, aligned=0)["kernel"] == (FEW if m <= 8 else TILES)


def test_the_rule_reaches_every_kernel_and_plan(lib):
    """Of each group, both widths of a unit and 1, 2 and 4 CTAs to a unit where there is no full round, 1 and 2 where there is."""
    seen = set()
    for n, k, group, m in _draws(60000, 1):
        p = _plan(lib, n, k, group, m)
        seen.add((group, p["kernel"]) if p["kernel"] != TC else (group, TC, p["tokens"], p["ranks"], p["rounds"]))
    for group in (32, 64, 128):
        assert {(group, FEW), (group, TILES)} <= seen
        for tokens in (32, 64):
            for ranks, rounds in ((1, 0), (2, 0), (4, 0), (1, 1), (2, 1)):
                assert (group, TC, tokens, ranks, rounds) in seen, (group, tokens, ranks, rounds)


def test_ctas_that_share_a_unit_divide_the_grid_and_all_have_work(lib):
    lib.ravel_debug_w4(TC)
    try:
        for n, k, group, m in _draws(20000, 2):
            if m <= 8:
                continue
            p = _plan(lib, n, k, group, m)
            units = -(-(-(-n // 32) * 2) // 8) * -(-m // p["tokens"])
            pieces = -(-(-(-k // 64)) // 2)
            assert p["kernel"] == TC and p["ranks"] in (1, 2, 4) and p["grid"] % p["ranks"] == 0 and 1 <= p["grid"] <= SMS
            assert p["ranks"] <= pieces and p["rounds"] == (units >= SMS)
            if not p["rounds"]:
                assert p["grid"] == units * p["ranks"]
            elif p["ranks"] > 1:   # each unit of the last round has its CTAs
                assert units % p["grid"] * p["ranks"] <= p["grid"] and units % p["grid"] > 0
    finally:
        lib.ravel_debug_w4(-1)


def test_a_choice_holds_for_its_thread_alone(lib):
    import threading
    own = _plan(lib, 128, 4096, 32, 16)["kernel"]
    lib.ravel_debug_w4(3 - own)
    try:
        assert _plan(lib, 128, 4096, 32, 16)["kernel"] == 3 - own
        there = []
        thread = threading.Thread(target=lambda: there.append(_plan(lib, 128, 4096, 32, 16)["kernel"]))
        thread.start()
        thread.join()
        assert there == [own]
    finally:
        lib.ravel_debug_w4(-1)
    assert _plan(lib, 128, 4096, 32, 16)["kernel"] == own
