"""CPU: what the nodes of a tree of new tokens see (csrc/pcs_attend_view.h) against
the definition, over random trees, rings, first tokens, windows, boxes and blocks
(tests/host/tree_check.cpp, built here with g++)."""
import os
import shutil
import subprocess

import pytest

from paper_2607_21686_gb300 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    gxx = shutil.which("g++")
    cuda = os.path.join(build._cuda_home(), "include")
    if not gxx or not os.path.exists(os.path.join(cuda, "cuda_runtime.h")):
        pytest.skip("no g++ or no CUDA headers")
    exe = str(tmp_path_factory.mktemp("tree") / "tree_check")
    subprocess.run([gxx, "-O2", "-std=c++17", "-fwrapv", "-I", build.CSRC, "-I", build.INCLUDE, "-I", cuda,
                    os.path.join(ROOT, "tests", "host", "tree_check.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_what_nodes_see(program, seed, kind):
    out = subprocess.run([program, str(seed), "1500", str(kind)], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr
