"""Which kernel a product of codes takes, asked of the library's own rule (csrc/lnmod_product_plan.hpp) on the CPU."""
import os
import subprocess

from paper_2605_17923_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
FEW, TILES, LARGE = 0, range(1, 9), 9


def program(folder):
    exe = os.path.join(str(folder), "product_plan_check")
    res = subprocess.run([build._hipcc(), "-std=c++17", "-O1", "-I", build.CSRC, "-I", build.INCLUDE,
                          os.path.join(HERE, "product_plan_check.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    return exe


def plans(problems, exe):
    """[(M, N, K, code, dtype)] -> [(kernel, whether the outputs stay in the caches)];  code "int8" or "e4m3", dtype "bf16" or "f32"."""
    lines = ["%d %d %d %d %d" % (M, N, K, code == "e4m3" and dtype == "f32", 2 if dtype == "bf16" else 4)
             for M, N, K, code, dtype in problems]
    run = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True)
    out = [tuple(int(v) for v in line.split()) for line in run.stdout.splitlines()]
    assert len(out) == len(problems)
    return [(k, bool(keep)) for k, keep in out]
