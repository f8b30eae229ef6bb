"""The example that trains a head against a collection and serves it beside the index."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2608_07152_gb300")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_train_head_finds_its_items():
    spec = importlib.util.spec_from_file_location(
        "train_head", os.path.join(ROOT, "examples", "train_head.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    r = mod.run(items_n=5000, steps=120, queries=40)
    # an untrained head's query has its item among 10 of 5,000 by chance (1 in 500)
    assert r["before"] <= 0.1
    assert r["last_loss"] < 0.5 * r["first_loss"]
    assert r["after"] >= 0.9
