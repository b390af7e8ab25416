"""The example that trains adapters beside a pruned layer and answers with them."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu


def test_training_lowers_the_error():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "adapters.py")
    spec = importlib.util.spec_from_file_location("adapters_example", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    before, after, single = example.run(120)
    assert all(map(math.isfinite, (before, after, single)))
    assert after < 0.5 * before and single < 2 * after + 1e-3
