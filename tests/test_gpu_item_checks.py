"""The checking build's work items of the MoE layer: one that its tables put outside the
arrays is latched as an error, and what the kernel still reads with it (its expert's
slot, its rows) lies inside."""
import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
EDEVICE = 6


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_04895_gb300 import build
    so = str(tmp_path_factory.mktemp("item") / "item_cases.so")
    subprocess.run([build.nvcc(), *build.ARCH, "-O3", "-std=c++17", "-shared", "-Xcompiler", "-fPIC",
                    "-DCRC_DEBUG", "-I", build.INCLUDE, "-I", build.CSRC, "--expt-relaxed-constexpr",
                    os.path.join(HERE, "item_cases.cu"), "-o", so], check=True)
    return ctypes.CDLL(so)


GOOD = dict(M=8, N=32, K=2, slots=4, slot0=3, count=1, tile_e=31, tile_row=4, tile_rows=12)


@pytest.mark.parametrize("wide", [0, 1])
@pytest.mark.parametrize("bad", [
    {}, dict(tile_e=32), dict(tile_e=127), dict(slot0=-1), dict(slot0=4), dict(tile_rows=0),
    dict(tile_rows=65), dict(tile_rows=13), dict(tile_row=5), dict(tile_row=65535), dict(count=0),
], ids=str)
def test_an_item_outside_the_arrays(lib, wide, bad):
    args = dict(GOOD, **bad)
    shared = torch.zeros(lib.item_bytes(), dtype=torch.uint8, device="cuda")
    t = torch.tensor([*args.values(), -7, -7, -7, -7], dtype=torch.int32, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert lib.item_run(wide, *(ctypes.c_void_p(x.data_ptr()) for x in (shared, t, err))) == 0
    ok, e, row0, rows = t[-4:].tolist()
    if not bad:
        assert (ok, e, row0, rows, int(err)) == (1, 31, 4, 12, 0)
        return
    assert ok == 0 and int(err) == EDEVICE
    assert (e, row0, rows) == (0, 0, 1)
