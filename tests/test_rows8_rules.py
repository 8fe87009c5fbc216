"""Rules of the operators on rows in 8 bits that choose a launch, on the host."""
import os
import shutil
import subprocess

import pytest

from paper_2609_16874_amd import build

SOURCE = r"""
#include <cstdio>
#include "rows8/rows.hpp"
int main()
{
    for (int dgamma = 0; dgamma < 2; dgamma++)
        for (int lanes : {8, 64, 256, 1024})
            for (int channels : {8, 1024, 16384})
                for (long long want : {1LL, 2LL, 8LL, 9LL, 300LL, 5000LL})
                    printf("%d %d %d %lld %d %d\n", dgamma, lanes, channels, want,
                           (int)cpe::rms_grad_blocks(want, channels, lanes, dgamma != 0),
                           (int)cpe::rms_most_blocks(channels));
}
"""


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_workgroups_of_the_norms_gradient(tmp_path):
    """One workgroup takes the turns of several only to spare dgamma's join: a
    gradient without dgamma has as many as its rows fill.  Never more than the
    scratch of partial sums has room for."""
    (tmp_path / "rule.hip").write_text(SOURCE)
    subprocess.run(["hipcc", "--offload-arch=gfx950", "--cuda-host-only", "-std=c++17", "-I", build.INCLUDE, "-I",
                    build.CSRC, "-o", str(tmp_path / "rule"), str(tmp_path / "rule.hip")], check=True, capture_output=True)
    lines = subprocess.run([str(tmp_path / "rule")], check=True, capture_output=True, text=True).stdout.splitlines()
    assert len(lines) == 2 * 4 * 3 * 6
    for line in lines:
        dgamma, lanes, channels, want, got, most = map(int, line.split())
        alone = dgamma and want <= (8 if lanes <= 64 else 1)
        assert got == (1 if alone else min(want, most)), line
