"""The operators and the optimizer together: the example's student learns."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_student_learns():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location(
        "distill_student", os.path.join(ROOT, "examples", "distill_student.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses = m.run(steps=60, tokens=300, hidden=100, inner=136, vocab=700, top=16, quiet=True)
    assert all(math.isfinite(v) for v in losses)
    assert sum(losses[-10:]) < 0.9 * sum(losses[:10])
    assert m.run(steps=8, tokens=300, hidden=100, inner=136, vocab=700, top=16,
                 quiet=True) == losses[:8]           # the same inputs, the same results
