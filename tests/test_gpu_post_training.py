"""The operators together, as examples/post_training.py runs them: delivery, scores, policy loss, gradients, step,
priorities."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "post_training.py")


def _example():
    spec = importlib.util.spec_from_file_location("post_training", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_post_training_iterations(capsys):
    out = _example().main(["--sequences", "6", "--max-len", "64", "--vocab", "3000", "--hidden", "96", "--steps", "4",
                           "--lr", "0.01", "--logits", "--preference"])
    losses = out["losses"]
    assert all(math.isfinite(x) for x in losses)
    # the first loss is that of the policy that acted (ratio 1, no divergence), and steps against the gradient lower it
    assert losses[1] < losses[0] and losses[-1] < losses[0]
    assert math.isfinite(out["preference"][0]) and out["preference"][3] == out["logits"][7] > 0
    assert out["logits"][1] == pytest.approx(losses[-1], abs=0.5)
