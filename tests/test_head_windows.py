"""What the products' loads into LDS address, replayed on the CPU
(tests/harness/head_windows.hip, host code alone): no lane reads past an array's end,
whatever the last part of a sum leaves of it."""
import os
import shutil
import subprocess

import pytest

HARNESS = os.path.join(os.path.dirname(os.path.abspath(__file__)), "harness", "head_windows.hip")


def _hipcc():
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    pytest.skip("hipcc not available")


def test_no_load_reads_past_an_arrays_end(tmp_path):
    exe = str(tmp_path / "head_windows")
    res = subprocess.run([_hipcc(), "--offload-host-only", "-std=c++17", "-O2", HARNESS, "-o", exe],
                         capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-4000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip() == "ok", run.stdout[-4000:] + run.stderr[-4000:]
