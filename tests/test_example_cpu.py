"""The example's models: every part of the parameters is stepped, once."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("name", ["Model", "GatedModel"])
def test_every_parameter_is_stepped_once(name):
    spec = importlib.util.spec_from_file_location("train_lm_step", os.path.join(ROOT, "examples", "train_lm_step.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    model = getattr(example, name)
    stepped = list(model.hidden) + list(model.others)
    assert sorted(stepped) == list(range(len(model.shapes)))
    assert all(rate > 0 for rate in model.others.values())
    assert all(min(model.shapes[i]) > 1 for i in model.hidden)       # the plan orthogonalises matrices
