"""The learner's operators together, as examples/grpo_update.py runs them: rollouts, advantages, loss, gradient, update, the next snapshot."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rewards_grow_and_snapshots_follow_the_learner():
    spec = importlib.util.spec_from_file_location("grpo_update", os.path.join(ROOT, "examples", "grpo_update.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    history, apart = example.main(updates=10, say=lambda *_: None)
    assert [h["version"] for h in history] == list(range(1, 11))
    assert all(np.isfinite([h["loss"], h["entropy"], h["grad_norm"]]).all() for h in history)
    # 64 answers of 32 tokens: the mean reward of a policy that has not moved is within 0.06 of one half (5 sigma)
    assert abs(history[0]["reward"] - 0.5) < 0.06 and history[-1]["reward"] > 0.6, [h["reward"] for h in history]
    # sampler (bf16 weights, half operands) and learner (f32 masters) under the same snapshot: the framework's own tolerance for a log-probability is 1e-2
    # against the same weights; master weights differ from their bf16 values by up to 2^-9 of themselves
    assert apart < 0.05 and all(h["largest_ratio"] < np.exp(0.05) for h in history)
