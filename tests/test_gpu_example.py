"""The post-training example runs end to end and learns: the reward doubles at
least, the preference loss falls from ln 2 (the policy is its own reference at
the start)."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_post_training_example(edp_lib):
    spec = importlib.util.spec_from_file_location(
        "post_training", os.path.join(ROOT, "examples", "post_training.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    h = example.train(40, log=lambda s: None)
    assert h["reward"][-1] > 2 * h["reward"][0] > 0
    assert abs(h["preference"][0] - math.log(2)) < 1e-5
    assert h["preference"][2] < h["preference"][1] < h["preference"][0]
    assert all(math.isfinite(x) for v in h.values() for x in v)
