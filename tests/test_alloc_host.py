"""C entries out of host memory: an error, no exception, no leak (no GPU)."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2608_23429_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
SOURCES = ["api.cpp", "cache.cpp", "table.cpp", "residual.cpp", "coded.cpp"]


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_out_of_host_memory(tmp_path):
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-g", "-O1"]
    inc = ["-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", os.path.join(ROCM, "include")]
    objs = []
    for src in SOURCES + ["host_stubs.cpp", "coded_check.cpp", "alloc_check.cpp"]:
        path = os.path.join(CSRC if src in SOURCES else HERE, src)
        objs.append(os.path.join(tmp_path, src + ".o"))
        other_main = ["-Dmain=coded_check_main"] if src == "coded_check.cpp" else []
        subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", *san, *inc, *other_main,
                        "-c", path, "-o", objs[-1]], check=True)
    exe = os.path.join(tmp_path, "alloc_check")
    libdir = os.path.join(ROCM, "lib")
    subprocess.run(["g++", *san, *objs, "-o", exe, "-L", libdir, "-lamdhip64",
                    f"-Wl,-rpath,{libdir}", "-lm"], check=True)
    env = dict(os.environ, TMPDIR=str(tmp_path),
               ASAN_OPTIONS="detect_leaks=1:abort_on_error=1:alloc_dealloc_mismatch=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "alloc ok" in r.stdout
