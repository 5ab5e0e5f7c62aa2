"""The launches of vq_cache_append over the whole range of batches, pages in 16 and in 8 bits (tests/host/append_launch_check.cpp).  No GPU needed; the
built libvq.so is what is tested."""
import os
import shutil
import subprocess

import pytest

import paper_2402_15319_amd as vq
from paper_2402_15319_amd import build as vqbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"), reason="needs g++ and the HIP headers")
def test_every_launch_is_one_that_the_runtime_takes(tmp_path):
    vq.lib()   # builds nothing: fails if the library is missing
    exe = tmp_path / "append_launch_check"
    cmd = ["g++", "-std=c++17", "-O1", "-rdynamic", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           os.path.join(ROOT, "tests", "host", "append_launch_check.cpp"), vqbuild.LIB_PATH,
           "-Wl,-rpath," + os.path.dirname(vqbuild.LIB_PATH), "-Wl,-rpath,/opt/rocm/lib", "-L/opt/rocm/lib", "-lamdhip64", "-o", str(exe)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout[-1000:] + res.stderr[-2000:]
    assert res.stdout.strip() == "append launches ok"
