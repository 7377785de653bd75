"""The example runs the solver and the losses together; each stage does what it is for."""
import importlib.util
import os

import pytest

import paper_2203_16340_amd as L

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_stage_improves_what_it_trains():
    spec = importlib.util.spec_from_file_location("preference_training", os.path.join(ROOT, "examples", "preference_training.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.run(vocab=1000, width=32, pairs=48, tokens=16)
    assert r["distill"][-1] < 0.5 * r["distill"][0]
    assert r["reward_status"] == L.CONVERGED and r["reward_right"] > 0.9
    assert abs(r["preference"][0] - 0.6931) < 1e-3 and r["preference"][-1] < 0.8 * r["preference"][0] and r["preference_right"] > 0.9
    assert max(r["policy"][-2:]) > r["policy"][0] + 0.1
