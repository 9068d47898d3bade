"""The example that runs the layer operators together, on a small model."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_prune_serve_recover():
    spec = importlib.util.spec_from_file_location("prune_serve_recover", os.path.join(ROOT, "examples", "prune_serve_recover.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    r = ex.run(tokens=8192, d=128, f=256, keep=100, vocab=500, swaps=30)
    before, after, accepted = r["search"]
    assert accepted > 0 and after < before
    dense, naive, pruned, served, trained = (r[k][0] for k in ("dense", "pruned, not refitted", "pruned", "pruned, 8 bits", "trained, not refitted"))
    assert dense < pruned < trained < 0.6 * naive      # the refit keeps most of the model, training gets part of it back
    assert abs(served - pruned) < 0.02 * pruned        # 8 bits cost next to nothing
