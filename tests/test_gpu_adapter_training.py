"""Adapters beside a compressed projection, trained and served as in examples/compressed_adapters.py."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_training_makes_up_for_the_compression():
    spec = importlib.util.spec_from_file_location("compressed_adapters", os.path.join(ROOT, "examples", "compressed_adapters.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.train(steps=120, tasks=2, rank=8, k=300, n=512, rows=128)
    # the adapters' space covers the inputs': more than half of the error goes, for every task and for served tokens
    assert all(after < 0.5 * before for before, after in zip(r["before"], r["after"])), r
    assert r["served"] < 0.5 * min(r["before"]), r
