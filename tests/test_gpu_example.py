"""The example that runs the operators around the step together: teacher in 4 bits, distillation, 4-bit AdamW, student in 4 bits."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "distill_and_serve.py")


def test_the_student_learns_and_serves_from_4_bits():
    spec = importlib.util.spec_from_file_location("distill_and_serve", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(steps=120)
    assert r["last"] < 0.7 * r["first"]      # learning, not a particular value
    assert r["cosine"] > 0.95                # 4-bit groups of 32: about 5 % of noise per matrix
