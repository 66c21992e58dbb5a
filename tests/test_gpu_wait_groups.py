"""Bounded waits of threads that go on together: when the wait runs out for some of them
only, all leave at the same place, and nobody is left at a barrier.  (The limits run
out by the test's own values; nothing faults or hangs.)"""
import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_04895_gb300 import build
    so = str(tmp_path_factory.mktemp("wait") / "wait_cases.so")
    subprocess.run([build.nvcc(), *build.ARCH, "-O3", "-std=c++17", "-shared", "-Xcompiler", "-fPIC",
                    "-I", build.INCLUDE, "-I", build.CSRC, "--expt-relaxed-constexpr",
                    os.path.join(HERE, "wait_cases.cu"), "-o", so], check=True)
    return ctypes.CDLL(so)


@pytest.mark.parametrize("threads,warps", [(256, 1), (256, 2), (96, 3), (256, 4), (256, 8),
                                           (512, 16), (1024, 32)])
def test_a_team_leaves_at_one_row(lib, threads, warps):
    rows, teams = 50, threads // (32 * warps)
    g = torch.Generator().manual_seed(threads + warps)
    for trial in range(40):
        give_up = torch.full((threads,), -1, dtype=torch.int32)
        want = torch.full((threads,), rows, dtype=torch.int32)
        for t in range(teams):
            if (trial + t) % 4 == 0:
                continue                                   # this team's rows all arrive
            mine = slice(32 * warps * t, 32 * warps * (t + 1))
            n = int(torch.randint(1, 32 * warps + 1, (1,), generator=g)) if trial % 2 else 1
            who = torch.randperm(32 * warps, generator=g)[:n]
            at = torch.randint(0, rows, (n,), dtype=torch.int32, generator=g)
            if trial % 3 == 0:                             # neighbouring rows
                at = at[0] + torch.arange(n, dtype=torch.int32) % 2
            give_up[mine][who] = at
            want[mine] = min(int(at.min()), rows)
        dev, left = give_up.cuda(), torch.full((threads,), -7, dtype=torch.int32, device="cuda")
        assert lib.row_team_run(threads, warps, rows, ctypes.c_void_p(dev.data_ptr()),
                                ctypes.c_void_p(left.data_ptr())) == 0
        assert torch.equal(left.cpu(), want)


@pytest.mark.parametrize("few", [0, 1, 16, 31, 32])
def test_a_warp_has_one_outcome(lib, few):
    def run(together):
        got = torch.full((32,), -7, dtype=torch.int32, device="cuda")
        assert lib.warp_wait_run(few, together, ctypes.c_void_p(got.data_ptr())) == 0
        return got.tolist()

    assert run(0) == [0] * few + [1] * (32 - few)          # each lane on its own: they part
    assert run(1) == [int(few == 0)] * 32
