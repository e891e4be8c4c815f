"""How many workgroups the norms between blocks launch at most (host code of csrc/launch_residual.h), against what the
compiler says of their kernels' registers: all of them are on the chip at once, and no more would be."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2001_04451_amd.build import COMMON_FLAGS, CSRC

PROGRAM = r"""
#include <cstdio>
#include "launch_residual.h"
int main() {
    for (int D : {8, 512, 520, 1024, 1032, 2048, 2056, 4096, 4104, 8192})
        std::printf("%d %d %d %d %d\n", D, lsh::residual_waves(D), lsh::residual_resident(lsh::kResidualFwd, D),
                    lsh::residual_resident(lsh::kResidualBwd, D), lsh::residual_resident(lsh::kResidualBwdPlain, D));
}
"""


def test_workgroups_are_those_that_fit(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc is missing")
    src, exe = str(tmp_path / "grid.cpp"), str(tmp_path / "grid")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.check_call([hipcc, *COMMON_FLAGS, src, "-o", exe])
    told = subprocess.run([hipcc, *COMMON_FLAGS, "--cuda-device-only", "-c", os.path.join(CSRC, "residual.hip"), "-o",
                           str(tmp_path / "residual.o"), "-Rpass-analysis=kernel-resource-usage"],
                          capture_output=True, text=True, check=True).stderr
    held = {}  # waves a SIMD holds: (fp32, plain or None, waves of a row)
    for name, body in re.findall(r"Function Name: (\S+)(.*?)LDS Size", told, flags=re.S):
        simd = int(re.search(r"Occupancy \[waves/SIMD\]: (\d+)", body).group(1))
        if m := re.search(r"residual_fwd_kernelILb([01])ELi(\d+)E", name):
            held[m[1], None, int(m[2])] = simd
        elif m := re.search(r"residual_bwd_kernelILb([01])ELb([01])ELi(\d+)E", name):
            held[m[1], m[2] == "1", int(m[3])] = simd
    assert len(held) == 30
    for line in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.splitlines():
        D, waves, *most = map(int, line.split())
        assert 256 * waves < D <= 512 * waves or (waves == 1 and D <= 512)
        for kind, n in zip((None, False, True), most):
            for f32 in "01":  # a workgroup: four waves, or those of a row
                assert n == 256 * (4 * held[f32, kind, waves] // max(4, waves)), (D, kind, f32)
