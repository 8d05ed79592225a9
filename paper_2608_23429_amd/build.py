"""Build step for libcheb.so (gfx950).

Host sources are compiled with amdclang++ as plain C++ against the HIP
runtime headers; the kernel source with hipcc for gfx950 only.  Packed fp32
instructions are disabled for all device code.  The library lands beside this
file, in-tree.
"""
import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libcheb.so")
BUILD_DIR = os.path.join(ROOT, "_build", "cheb")

ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
ARCH = "gfx950"

HOST_SOURCES = ["api.cpp", "cache.cpp", "table.cpp", "residual.cpp", "coded.cpp",
                "norm.cpp"]
DEVICE_SOURCES = ["kernels.hip", "predict_coded.hip", "norm.hip", "coded.hip"]

DEVICE_FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument", "-fvisibility=hidden",
]
HOST_FLAGS = [
    "-O2", "-std=c++17", "-fPIC", "-Wall", "-Wextra", "-D__HIP_PLATFORM_AMD__",
    "-fvisibility=hidden",
]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines()
                    if "packed-fp32-ops' is not a recognized feature" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"command failed ({r.returncode}): {' '.join(cmd)}\n{out}")
    if verbose and out.strip():
        print(out, flush=True)


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    hipcc = os.path.join(ROCM, "bin", "hipcc")
    cxx = os.path.join(ROCM, "llvm", "bin", "clang++")
    if not os.path.exists(cxx):
        cxx = shutil.which("g++") or "g++"
    incs = ["-I", INCLUDE, "-I", CSRC, "-I", os.path.join(ROCM, "include")]
    cmds, objs = [], []
    for compiler, sources in ([hipcc, *DEVICE_FLAGS], DEVICE_SOURCES), ([cxx, *HOST_FLAGS],
                                                                        HOST_SOURCES):
        for src in sources:
            objs.append(os.path.join(BUILD_DIR, src + ".o"))
            cmds.append([*compiler, *incs, "-c", os.path.join(CSRC, src), "-o", objs[-1]])
    with ThreadPoolExecutor(max_workers=4) as pool:   # the kernel sources take a minute or two each
        list(pool.map(lambda cmd: _run(cmd, verbose), cmds))
    tmp = LIB + ".tmp"
    _run([hipcc, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs,
          "-Wl,--no-undefined", "-Wl,-soname,libcheb.so"], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-q" not in sys.argv))
