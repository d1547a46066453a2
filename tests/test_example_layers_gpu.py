"""The example that trains, stores, answers and verifies with 4-bit layers, as a user runs it."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_store_verify.py")


def test_train_store_verify():
    spec = importlib.util.spec_from_file_location("train_store_verify", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.main(["--steps", "40", "--inputs", "32"])
    assert r["loss"][1] < 0.5 * r["loss"][0]
    assert r["accuracy"] >= 0.9
    assert r["bounds hold"]
    assert r["verified"] + r["attacked"] <= 1.0   # no input is both
