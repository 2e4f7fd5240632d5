"""The example that runs the operators beside the scoring step together: a model writes, a smaller one learns from it."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "write_and_learn.py")


def test_the_student_learns_what_the_teacher_writes():
    spec = importlib.util.spec_from_file_location("write_and_learn", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    r = module.main(words=1500, hidden=64, sentences=32, length=12, passes=25)
    assert r["text"].shape == (13, 32) and len(np.unique(r["text"])) > 20
    # an untrained output layer gives every word 1 / V; a learned one has to be nearer to the teacher than to that
    assert abs(r["untrained"] + np.log(1500)) < 1e-3
    assert r["losses"][-1] < r["losses"][0] and r["student"] > 0.5 * (r["teacher"] + r["untrained"])
    again = module.main(words=1500, hidden=64, sentences=32, length=12, passes=2)
    assert np.array_equal(again["text"], r["text"]) and again["losses"][:2] == pytest.approx(r["losses"][:2], rel=1e-5)
