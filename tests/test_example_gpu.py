"""The example that runs the training operators together learns."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu


def test_a_student_learns_from_an_aligned_teacher():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "aligned_distillation.py")
    spec = importlib.util.spec_from_file_location("aligned_distillation", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    history = example.train(steps=40)
    assert all(math.isfinite(v) for step in history for v in step)
    assert history[-1][0] < 0.5 * history[0][0]  # the divergence falls
    assert history[-1][1] > history[0][1] + 1.0  # and the wrong alignments come to cost more than the right ones
