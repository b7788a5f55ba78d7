"""The example of a whole actor update learns."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "actor_update.py")


def test_actor_update_learns():
    """A response's even share starts at about one half, with a deviation of 0.5 / sqrt(64 * 16) = 0.016 of an iteration's mean:
    ten of them above 0.6 are not chance."""
    spec = importlib.util.spec_from_file_location("actor_update", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    rewards, norm = mod.train(40)
    assert abs(rewards[0] - 0.5) < 0.1 and np.mean(rewards[-10:]) > 0.6
    assert np.isfinite(norm) and norm > 0
