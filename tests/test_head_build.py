"""Properties of the head operators' device code that the compiler reports
without a GPU."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_16874_amd import build


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_dynamic_lds_holds_doubles(tmp_path):
    """The join of partial results keeps 64-bit sums in the norm's dynamic LDS,
    whose declared alignment the compiler takes for granted."""
    out = tmp_path / "norm.ll"
    flags = [f for f in build.HIPCC_FLAGS if f != "-O3"]
    subprocess.run(["hipcc", *flags, "-O1", "--cuda-device-only", "-S", "-emit-llvm", "-I", build.INCLUDE, "-I",
                    build.CSRC, "-o", str(out), os.path.join(build.CSRC, "head", "norm_f32.hip")],
                   check=True, capture_output=True)
    found = re.findall(r"external .*addrspace\(3\) global \[0 x float\].*align (\d+)", out.read_text())
    assert found and all(int(a) >= 8 for a in found), found
