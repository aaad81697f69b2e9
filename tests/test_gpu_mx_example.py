"""The example runs the MX operators together: training with 8-bit checkpoints and accumulated gradients, serving token by token."""
import importlib.util
import os

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


def test_training_and_serving():
    spec = importlib.util.spec_from_file_location("mx_layer_example", os.path.join(ROOT, "examples", "mx_layer.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    lines = []
    r = example.main(["--steps", "120", "--tokens", "512"], report=lines.append)
    assert r["mx"] < 0.35 * r["before"]       # it learns: a broken gradient leaves the loss where it was, or sends it up
    assert r["fp32"] < r["mx"]                # and 4 bits cost something
    assert r["apart"] < 5e-4                  # a token's blocks are its own: the batch changes no code of the first layer, rounding of sums hardly one of the second
    assert len(lines) >= 3
