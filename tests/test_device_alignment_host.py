"""The kernels' wide loads and stores say the alignment that their addresses
have (no GPU: the compiler's own check, nothing is generated)."""
import os
import shutil
import subprocess

import pytest

from paper_2608_23429_amd import build

HIPCC = os.path.join(build.ROCM, "bin", "hipcc")


@pytest.mark.skipif(not os.path.exists(HIPCC) and shutil.which("hipcc") is None,
                    reason="needs hipcc")
@pytest.mark.parametrize("source", build.DEVICE_SOURCES)
def test_no_pointer_claims_more_alignment(source):
    flags = [f for f in build.DEVICE_FLAGS if f != "-O3"]
    r = subprocess.run([HIPCC if os.path.exists(HIPCC) else "hipcc", *flags,
                        "-Werror=align-mismatch", "-fsyntax-only", "--cuda-device-only",
                        "-I", build.INCLUDE, "-I", build.CSRC, os.path.join(build.CSRC, source)],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
