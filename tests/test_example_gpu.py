"""examples/teach_a_student.py runs the norm, the losses and the sample layer together, and learns."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_an_ensemble_learns_and_teaches():
    spec = importlib.util.spec_from_file_location("teach_a_student", os.path.join(ROOT, "examples", "teach_a_student.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.main(steps=40)
    assert got["ensemble"][1] < 0.5 * got["ensemble"][0]
    assert got["student"][1] < 0.5 * got["student"][0]
    assert got["agree"] > 0.5
