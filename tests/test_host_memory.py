"""CPU: attention over 8-bit caches where working memory cannot be had (csrc/pcs_attend.cpp
over stand-ins, tests/host/memory_check.cpp, built here with g++)."""
import os
import shutil
import subprocess

import pytest

from paper_2607_21686_gb300 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_attention_does_without_memory_it_need_not_have(tmp_path):
    gxx = shutil.which("g++")
    cuda = os.path.join(build._cuda_home(), "include")
    if not gxx or not os.path.exists(os.path.join(cuda, "cuda_runtime.h")):
        pytest.skip("no g++ or no CUDA headers")
    exe = str(tmp_path / "memory_check")
    subprocess.run([gxx, "-O1", "-std=c++17", "-I", build.CSRC, "-I", build.INCLUDE, "-I", cuda,
                    os.path.join(ROOT, "tests", "host", "memory_check.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr
