"""examples/distill_step.py: the operators around the output layer together, on small sizes."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "distill_step.py")


def test_student_approaches_its_teacher():
    spec = importlib.util.spec_from_file_location("distill_step", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, (teacher, student, plain) = example.train(tokens=256, features=256, vocab=1000, rank=8, top=16, steps=40)
    print(losses[0], losses[-1], teacher, student, plain, flush=True)
    assert all(math.isfinite(x) for x in losses)
    # the adapter has the teacher's rank, so most of what separates the two can be learnt
    assert losses[-1] < 0.75 * losses[0]
    assert abs(student - teacher) < abs(plain - teacher)
