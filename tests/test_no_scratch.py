"""The kernels that keep matrix accumulators in registers over divergent code spill none of them: a
variant that did gave wrong sums in the lanes that had taken another branch."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_21135_amd", "csrc")


@pytest.mark.parametrize("name", ["qattend.hip", "qcache.hip", "verify.hip"])
def test_kernels_use_no_scratch_memory(name):
    from paper_2503_21135_amd import build
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    cmd = [build.HIPCC] + build.FLAGS + ["--cuda-device-only", "-S", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                                         os.path.join(CSRC, name), "-o", "-"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    sizes = re.findall(r"^\s*\.private_segment_fixed_size:\s*(\d+)", res.stdout, re.M)
    assert len(sizes) > 3 and set(sizes) == {"0"}
