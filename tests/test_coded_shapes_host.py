"""Launch shapes of calls over 8-bit entries, built for the host.  CPU only."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_coded_shapes(tmp_path):
    exe = os.path.join(tmp_path, "coded_shapes_check")
    subprocess.run(["g++", "-std=c++17", "-O2", "-D__HIP_PLATFORM_AMD__", "-I",
                    os.path.join(ROOT, "paper_2608_23429_amd", "csrc"), "-I",
                    os.path.join(ROOT, "include"), "-I", os.path.join(ROCM, "include"),
                    os.path.join(HERE, "coded_shapes_check.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "coded_shapes ok" in r.stdout
