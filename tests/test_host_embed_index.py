"""The embedding gradient's index arithmetic at up to 2^31 - 1 tokens (tests/host_embed_index_check.cpp).  CPU only."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(HERE, "host_embed_index_check.cpp")


def test_pieces_and_spans(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "host_embed_index_check")
    # (signed overflow ends the program)
    res = subprocess.run([hipcc, "-x", "hip", "--cuda-host-only", "-std=c++17", "-O1", "-ftrapv", SRC, "-o", exe,
                          "-Wl,--unresolved-symbols=ignore-in-object-files"], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "0 failure(s)" in run.stdout, (run.returncode, run.stdout[-3000:], run.stderr[-3000:])
