"""The example that runs the context cache's operators together: prompts, decoded
tokens, eviction and the rolling step that reads what stays."""
import importlib.util
import os

import numpy as np
import pytest

import synth
from oracle import expert

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_34170_gb300 import build, load
    build.build()
    load()
    spec = importlib.util.spec_from_file_location("vlm_prefix", os.path.join(ROOT, "examples", "vlm_prefix.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_prefix_to_rolling_step(example):
    got = example.main(["--robots", "3", "--prompt", "90", "--decode", "5", "--keep", "40", "--layers", "2"])
    again = example.main(["--robots", "3", "--prompt", "90", "--decode", "5", "--keep", "40", "--layers", "2"])
    assert torch.equal(got["tokens"], again["tokens"]) and torch.equal(got["released"], again["released"])
    for kept, length in zip(got["kept"], [got["lengths"]] * 2):
        for b in range(3):
            index = kept[b, 0].cpu().numpy()
            assert (np.diff(index) > 0).all() and list(index[:4]) == [0, 1, 2, 3]
            assert list(index[-5:]) == list(range(int(length[b]) - 5, int(length[b])))
    # every query's weights sum to one: its heads over every call's queries
    total = got["mass"].sum(-1)
    queries = got["lengths"].float() * 8      # the prompt's tokens and the decoded ones, 8 heads
    assert torch.allclose(total, queries[None, :, None].expand_as(total), rtol=1e-3)
    # the step reads the context that was read back: the oracle's released actions for it
    cfg = got["cfg"]
    k, v = (x.float().cpu().numpy() for x in got["context"])
    seeds = synth.robot_seeds(7, 3)
    buffer, counters = expert.reset(cfg, seeds)
    want, *_ = expert.roll_step(cfg, synth.make_weights(cfg), buffer, synth.staggered_times(cfg.slots), k, v, k.shape[3],
                                np.zeros((3, 0, cfg.width), np.float32), synth.make_delta(3, 2, cfg.slots), seeds, counters)
    assert np.abs(got["released"].cpu().numpy() - want).max() <= 5e-2
