"""CPU: what the operators over a paged cache refuse, and which kernels they choose
(csrc/pcs_attend.cpp), over stand-ins for a context and for the launches
(tests/host/refuse_check.cpp, built here with g++)."""
import os
import shutil
import subprocess

import pytest
import torch

from paper_2607_21686_gb300 import build, pcs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_refusals(tmp_path):
    gxx = shutil.which("g++")
    cuda = os.path.join(build._cuda_home(), "include")
    if not gxx or not os.path.exists(os.path.join(cuda, "cuda_runtime.h")):
        pytest.skip("no g++ or no CUDA headers")
    exe = str(tmp_path / "refuse_check")
    subprocess.run([gxx, "-O1", "-std=c++17", "-I", build.CSRC, "-I", build.INCLUDE, "-I", cuda,
                    os.path.join(ROOT, "tests", "host", "refuse_check.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr


def test_row_bytes():
    for heads, dim in ((1, 16), (16, 64), (8, 128), (3, 80), (31, 64)):
        n = pcs.kv_row_bytes(heads, dim)
        assert n % 32 == 0 and heads * dim + heads <= n < heads * dim + heads + 32


def test_pools_of_codes_agree():
    k = torch.zeros(4, 16, 160, dtype=torch.uint8)
    t = torch.zeros(2, 2, dtype=torch.int32)
    for args, kw in (((k, k, t), dict(codes=torch.float8_e4m3fn, heads=2, head_dim=64)),):
        with pytest.raises(ValueError):  # not on a GPU
            pcs.KvCache(*args, **kw)
