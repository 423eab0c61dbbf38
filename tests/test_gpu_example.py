"""The example that runs the largest logits, cross entropy and distillation together, at a small size."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_a_role_is_taught_by_another():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "teach_role.py")
    spec = importlib.util.spec_from_file_location("teach_role", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    out = example.main(["--steps", "40", "--rows-per-turn", "24", "--vocabulary", "1001", "--top", "16"])
    assert out["warm"][-1] < out["warm"][0]
    assert out["distill"][-1] < out["distill"][0]
    assert out["last"][0] < 0.5 * out["first"][0]
    token, p = out["answer"]
    assert 0 <= token < 1001 and 0.0 < p <= 1.0
