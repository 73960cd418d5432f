"""The long-context example runs, and its parts agree with each other."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_long_context_example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import long_context
    r = long_context.main()
    # bf16 states through four layers, rounded at different places
    assert r["parallel_vs_steps"] < 3e-2
    assert r["prefix_vs_decode"] < 1e-2  # two roundings of bf16 outputs
    assert r["weight_per_head"] < 1e-5
    assert r["cut"] == (184, 96) and r["slots_now"] == 96 + 16
    assert r["position"] == long_context.PROMPT + 40 + 48 and r["finite"]
