"""How the operators around the step cut their work up: the library's host code with a stand-in for the HIP runtime
(tests/host_training_check.cpp).  CPU only."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(HERE, "host_training_check.cpp")


def test_pieces_workspaces_and_grids(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "host_training_check")
    res = subprocess.run([hipcc, "-x", "hip", "--cuda-host-only", "-std=c++17", "-O1", "-g", "-Xarch_host", "-fsanitize=address",
                          SRC, "-o", exe, "-Wl,--unresolved-symbols=ignore-in-object-files"], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert run.returncode == 0 and "0 failure(s)" in run.stdout, (run.stdout[-3000:], run.stderr[-3000:])
