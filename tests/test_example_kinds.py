"""What the example of an actor update refuses, before it needs a GPU."""
import importlib.util
import os

import pytest

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "actor_update.py")


@pytest.mark.parametrize("kind", ["policies", "", None])
def test_losses_that_the_example_does_not_know(kind):
    spec = importlib.util.spec_from_file_location("actor_update", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    with pytest.raises(ValueError, match="grpo, policy, preference"):
        mod.train(1, kind=kind)
