"""The example that quantises a layer, tunes two adapters beside it and serves both: the operators working together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_adapters_learn_what_quantisation_lost():
    spec = importlib.util.spec_from_file_location("tune_adapters", os.path.join(ROOT, "examples", "tune_adapters.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, ids, served = example.main(verbose=False)
    assert losses[-1] < 0.9 * losses[0]
    adapted = max(e for a, e in zip(ids, served) if a >= 0)
    assert adapted < 1.0 and all(e == e for e in served)
