"""The checking flavour of the library on the MoE layer: every item's tile, rows, expert
and slot are checked before use; the error word stays zero and every output equals
the product library's."""
import os
import subprocess
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))


def test_checking_build_runs_clean_and_equals_the_product(tmp_path):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_04895_gb300 import build
    build.build()
    build.build(debug=True)
    out = tmp_path / "debug.npz"
    r = subprocess.run([sys.executable, os.path.join(HERE, "operator_debug_cases.py"), str(out)],
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    dbg = dict(np.load(out))
    import paper_2609_04895_gb300 as P
    sys.path.insert(0, HERE)
    try:
        import operator_debug_cases
    finally:
        sys.path.remove(HERE)
    rel = operator_debug_cases.run_cases(P)
    assert set(dbg) == set(rel) and len(rel) > 1
    for k in rel:
        assert np.array_equal(dbg[k], rel[k]), k
    assert int(rel["error"]) == 0
