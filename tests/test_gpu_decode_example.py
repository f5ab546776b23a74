"""The VLM example with rotary positions, 4-bit weights and drawn tokens: it runs, repeats, and what it hands to
the rolling step is what the step reads."""
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


@pytest.mark.parametrize("more", [["--rotary"], ["--four-bit"], ["--temperature", "0.7"], ["--rotary", "--four-bit", "--temperature", "0.7"]])
def test_decoding_with_them_reaches_the_rolling_step(example, more):
    args = ["--robots", "3", "--prompt", "90", "--decode", "5", "--keep", "40", "--layers", "2"] + more
    got, again = example.main(args), example.main(args)
    for name in ("tokens", "released", "lengths"):
        assert torch.equal(got[name], again[name])
    assert ((got["tokens"] >= 0) & (got["tokens"] < 512)).all()
    cfg = got["cfg"]
    k, v = (x.float().cpu().numpy() for x in got["context"])
    seeds = synth.robot_seeds(7, 3)
    buffer, counters = expert.reset(cfg, seeds)
    want, *_ = expert.roll_step(cfg, synth.make_weights(cfg), buffer, synth.staggered_times(cfg.slots), k, v, k.shape[3],
                                np.zeros((3, 0, cfg.width), np.float32), synth.make_delta(3, 2, cfg.slots), seeds, counters)
    assert np.abs(got["released"].cpu().numpy() - want).max() <= 5e-2
