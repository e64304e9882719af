"""The example that runs the worker-side operators and the group update together: it learns."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_workers_learn():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "language_model_workers.py")
    spec = importlib.util.spec_from_file_location("language_model_workers", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    rewards, losses = example.main(30)
    assert rewards[0] < 0.12 and sum(rewards[-3:]) / 3 > 2 * rewards[0]      # one token in 16 is good to begin with
    assert abs(losses[0] - 0.6931) < 1e-3                                    # the policy is its own reference: log 2
    assert losses[-1] < 0.6 * losses[0]
