"""Launch shapes and grids of the operators that hold activations in 8 bits, checked without a GPU: every hidden size, from one
row to the largest number of them."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = next((c for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")) if c and os.path.exists(c)), None)


@pytest.mark.skipif(HIPCC is None, reason="hipcc not found")
def test_launches(tmp_path):
    exe = str(tmp_path / "code_launch_check")
    build = subprocess.run([HIPCC, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2605_17923_amd", "csrc"), "-I",
                            os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "code_launch_check.cpp"), "-o", exe],
                           capture_output=True, text=True)
    assert build.returncode == 0, build.stdout + build.stderr
    run = subprocess.run([exe], capture_output=True, text=True)
    assert run.returncode == 0 and run.stdout.startswith("0 failures"), run.stdout + run.stderr
