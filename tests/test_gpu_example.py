"""The example that runs the norm, the MoE layer and the 8-bit rows beside the cache."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_decode_from_slots_equals_decode_with_every_expert():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_04895_gb300 import build
    build.build()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import decode_from_slots as ex
    finally:
        sys.path.pop(0)
    r = ex.run(tokens=40, seed=3)
    assert r["same"] and r["finite"] and r["error"] == 0
    assert r["copies"] == r["planned"] > 0
    assert 0.0 < r["hit"] < 1.0
