"""hipcc's resource report for the kernels of the row codes, their product and the rotations: none has scratch, but for a few
registers of row norms in bf16 (measured with them: a wave more on a SIMD, or four units a lane, are worth more), and for fp32 rows
of more than 32 rounds of heads, which eight waves hold with eight units a lane.  Needs only hipcc."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2605_17923_amd import build

ALLOWED = {r"rotary_fwd_kernel<lnmod::bf16_io, 1, (true|false), 3>": 12, r"rotary_bwd_kernel<lnmod::bf16_io, 1, (true|false), 4>": 32,
           r"rotary_bwd_kernel<lnmod::f32_io, 1, (true|false), 8>": 236}


def test_no_scratch(tmp_path):
    if shutil.which(build._hipcc()) is None and not os.path.exists(build._hipcc()):
        pytest.skip("hipcc not found")

    def report(src):
        cmd = [build._hipcc()] + build.HIPCC_FLAGS + ["-Rpass-analysis=kernel-resource-usage", "-c", os.path.join(build.CSRC, src), "-o",
                                                       os.path.join(str(tmp_path), src + ".o")]
        res = subprocess.run(cmd, capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-2000:]
        return res.stderr

    with ThreadPoolExecutor(max_workers=2) as pool:
        text = "\n".join(pool.map(report, ["lnmod_product.hip", "lnmod_rotary.hip", "lnmod_rowcodes.hip"]))
    names = re.findall(r"Function Name: (\S+)", text)
    scratch = [int(v) for v in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", text)]
    assert len(names) == len(scratch) and len(names) > 100
    plain = subprocess.run(["c++filt"], input="\n".join(names), capture_output=True, text=True, check=True).stdout.splitlines()
    for name, bytes_ in zip(plain, scratch):
        most = max([v for k, v in ALLOWED.items() if re.search(k, name)], default=0)
        assert bytes_ <= most, "%s spills %d bytes per lane" % (name, bytes_)
