"""Which values threads lay out for the gated block's tiled products, on the host
(tests/fake_hip/stage_places.cpp)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_places_of_values_that_are_laid_out(tmp_path):
    """Also of the workgroups that a rounded-up grid has past the last array's."""
    from paper_2101_08763_amd import build as B
    if not os.path.exists(B.HIPCC):
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "stage_places")
    r = subprocess.run([B.HIPCC, "-O1", "-std=c++17", f"-I{B.INCLUDE}", f"-I{B.CSRC}", f"--offload-arch={B.ARCH}", "-x", "hip",
                        os.path.join(ROOT, "tests", "fake_hip", "stage_places.cpp"), "-o", exe],
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "checks passed" in r.stdout, r.stdout + r.stderr
