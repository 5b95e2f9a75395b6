"""The scales and biases that a product's waves read lie inside their arrays, also for waves whose part of a tile is beyond the last
row or feature: a small C++ program walks every wave of every tile shape at sizes that end inside a tile, with the index functions
of the kernels.  Needs only hipcc's host compiler."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2605_17923_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_every_index_is_inside(tmp_path):
    if shutil.which(build._hipcc()) is None and not os.path.exists(build._hipcc()):
        pytest.skip("hipcc not found")
    exe = str(tmp_path / "product_reads_check")
    res = subprocess.run([build._hipcc(), "-std=c++17", "-O1", "-I", build.CSRC, "-I", build.INCLUDE,
                          os.path.join(HERE, "product_reads_check.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    run = subprocess.run([exe], capture_output=True, text=True)
    sys.stdout.write(run.stdout)
    assert run.returncode == 0, run.stdout
