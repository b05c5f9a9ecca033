"""The example that trains a classifier on features and serves it from 8 bits, end to end."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("state_bits", [8, 32])
def test_classifier_learns_and_is_served(state_bits):
    spec = importlib.util.spec_from_file_location("softmax_classifier", os.path.join(ROOT, "examples", "softmax_classifier.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.run(classes=6, n_train=600, n_test=200, steps=120, state_bits=state_bits, say=lambda text: None)
    assert abs(r["first_loss"] - 1.791759) < 1e-4                # log 6: all weights zero
    assert r["last_loss"] < 0.5 * r["first_loss"] and r["accuracy"] > 0.6
    assert r["accuracy_int8"] > r["accuracy"] - 0.03 and r["one_at_a_time"]
    # codes are within half a step, 1/254 of a row's largest, and rows have norm 1: Phi_x Phi_y is off by at most
    # 2 (1/254) sqrt(385), and the product of two such errors
    assert r["kernel_error"] < 2 * 385 ** 0.5 / 254 + 385 / 254 ** 2
