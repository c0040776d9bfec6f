"""The example's arguments (no GPU needed)."""
import importlib.util
import os

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_rate_of_zero_is_a_rate():
    spec = importlib.util.spec_from_file_location("refit_layernorm_arguments", os.path.join(ROOT, "examples", "refit_layernorm.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    assert ex.filter_rate(0.0, "muon") == 0.0 and ex.filter_rate(0.1, "sgd") == 0.1
    assert ex.filter_rate(None, "muon") == 0.4 and ex.filter_rate(None, "sgd") == 0.0005
