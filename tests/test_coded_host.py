"""Histories of 8-bit entries without a GPU: the library's host code built
with g++ under AddressSanitizer and UndefinedBehaviorSanitizer, with launchers
that work on host memory, and the Python face's refusals."""
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import coded_ref as ref
import paper_2608_23429_amd as cheb

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2608_23429_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
SOURCES = ["api.cpp", "cache.cpp", "table.cpp", "residual.cpp", "coded.cpp"]


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_coded_ring_under_asan_ubsan(tmp_path):
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
           "-fno-omit-frame-pointer", "-g", "-O1"]
    inc = ["-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", os.path.join(ROCM, "include")]
    objs = []
    for src in SOURCES + ["host_stubs.cpp", "coded_check.cpp"]:
        path = os.path.join(CSRC if src in SOURCES else HERE, src)
        objs.append(os.path.join(tmp_path, src + ".o"))
        subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", *san, *inc, "-c", path,
                        "-o", objs[-1]], check=True)
    exe = os.path.join(tmp_path, "coded_check")
    libdir = os.path.join(ROCM, "lib")
    subprocess.run(["g++", *san, *objs, "-o", exe, "-L", libdir, "-lamdhip64",
                    f"-Wl,-rpath,{libdir}", "-lm"], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "coded ok" in r.stdout


@pytest.mark.parametrize("layout", ["slots", "interleaved"])
@pytest.mark.parametrize("quant", ["mxint8", "mxfp8"])
def test_layout(quant, layout):
    sizes = [5, 0, 4097, 1, 4096]
    codes = {"mxint8": cheb.CHEB_QUANT_MXINT8, "mxfp8": cheb.CHEB_QUANT_MXFP8}
    kinds = {"slots": cheb.CHEB_LAYOUT_SLOTS, "interleaved": cheb.CHEB_LAYOUT_INTERLEAVED}
    lay = cheb.cheb_cache_layout_quant(3, cheb.CHEB_BF16, codes[quant], sizes, kinds[layout])
    off, size = ref.offsets(sizes)
    assert list(lay["seg_offset"]) == off and lay["slot_numel"] == size
    assert lay["arena_bytes"] >= 3 * size * 33 // 32


def test_python_refusals():
    with pytest.raises(cheb.ChebError) as e:
        cheb.ChebCache(2, torch.bfloat16, [64], device="cpu", quant="int4")
    assert e.value.name == "CHEB_E_INVAL"
    with pytest.raises(cheb.ChebError) as e:       # the arena is GPU memory
        cheb.ChebCache(2, torch.bfloat16, [64], device="cpu", quant="mxint8")
    assert e.value.name == "CHEB_E_INVAL"
    with pytest.raises(cheb.ChebError) as e:
        cheb.cheb_cache_layout_quant(2, cheb.CHEB_BF16, 0, [64], 0)
    assert e.value.name == "CHEB_E_INVAL"


def test_reference_formats():
    """The definition itself: error bounds, ties, the choice of exponent."""
    rng = np.random.default_rng(3)
    x = rng.normal(size=(512, 32)) * np.exp(rng.normal(size=(512, 1)) * 5)
    x = x.astype(np.float32).astype(np.float64)
    for quant, limit in (("mxint8", 127 / 64), ("mxfp8", 448.0)):
        q, e, finite = ref.groups(x, quant)
        top = np.abs(x).max(1)
        assert finite.all() and (top <= limit * 2.0 ** e).all()
        assert (top > limit * 2.0 ** (e - 1)).all()
        off = np.abs(ref.held(x, quant).reshape(x.shape) - x)
        if quant == "mxint8":
            assert (off <= np.ldexp(1.0, e - 7)[:, None]).all()
            assert (off <= top[:, None] / 126).all()
        else:
            assert (off <= np.maximum(np.abs(x) / 16, np.ldexp(1.0, e - 10)[:, None])).all()
    assert list(ref.near_e4m3(np.array([17.0, 19.0, 464.0, 2.0 ** -10, 3 * 2.0 ** -10]))) == [
        16.0, 20.0, 448.0, 0.0, 2.0 ** -8]
