"""CPU check of the chunk prefill's ring depth (MTN_PF_STAGES, a tuning define of
the build): a depth that leaves one of the kernel's forms a negative number of
copies to wait for does not compile."""
import os
import subprocess

import pytest

from paper_2607_02640_amd import build

SRC = os.path.join(build.CSRC, "mtn_kernels.hip")


@pytest.mark.parametrize("stages,fits", [(3, False), (4, False), (5, True), (8, True), (9, False)])
def test_ring_depth(stages, fits):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    r = subprocess.run([build.HIPCC, *build.compile_flags("mtn_kernels.hip"), f"-DMTN_PF_STAGES={stages}",
                        "--cuda-device-only", "-fsyntax-only", SRC], capture_output=True, text=True)
    assert (r.returncode == 0) == fits, r.stderr[-2000:]
    assert fits or "ring depth" in r.stderr
