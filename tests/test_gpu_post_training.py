"""The post-training example: losses fall, every rollout's gradient is most like itself."""
import importlib.util
import os

import pytest
import torch

from tests._util import say

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example_runs_and_learns():
    spec = importlib.util.spec_from_file_location("post_training", os.path.join(ROOT, "examples", "post_training.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    say("case: post-training example")
    out = m.main()
    assert out["policy"][-1] < out["policy"][0] - 0.1
    assert out["preference"][-1] < out["preference"][0] - 0.1
    assert torch.isfinite(out["head"]).all()
    assert (out["index"][:, 0] == torch.arange(m.N)).all() and (out["score"][:, 0] - 1).abs().max() < 1e-4
    again = m.main()
    assert torch.equal(out["head"], again["head"]) and out["policy"] == again["policy"]
