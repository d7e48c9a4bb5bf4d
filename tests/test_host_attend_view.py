"""CPU: the arithmetic by which the attention kernels know what each new token
sees (csrc/pcs_attend_view.h) against the definition, token by token, over
random rings, first tokens, windows, boxes and blocks of rows
(tests/host/view_check.cpp, built here with g++)."""
import os
import shutil
import subprocess

import pytest

from paper_2607_21686_gb300 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def checker(tmp_path_factory):
    gxx = shutil.which("g++")
    cuda = os.path.join(build._cuda_home(), "include")
    if not gxx or not os.path.exists(os.path.join(cuda, "cuda_runtime.h")):
        pytest.skip("no g++ or no CUDA headers")
    exe = str(tmp_path_factory.mktemp("view") / "view_check")
    subprocess.run([gxx, "-O2", "-std=c++17", "-fwrapv", "-I", build.CSRC, "-I", build.INCLUDE, "-I", cuda,
                    os.path.join(ROOT, "tests", "host", "view_check.cpp"), "-o", exe], check=True)
    return exe


def run(checker, *args):
    out = subprocess.run([checker] + [str(x) for x in args], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr


@pytest.mark.parametrize("sinks,ring,box", [(100, 64, 16), (4, 1024, 128), (4, 64, 16), (64, 128, 128), (16, 203, 8),
                                            (1, 100, 64), (130, 150, 32)])
@pytest.mark.parametrize("group", [1, 4])
def test_first_tokens_of_a_block_that_laps_its_ring(checker, sinks, ring, box, group):
    # Rows at first positions see no first token ahead of themselves.
    for beyond in (1, 6, box // 2, box, box + 1, 2 * box + 3):
        n = sinks + ring + beyond
        run(checker, sinks, ring, 0, n, n, box, group, 0)
        run(checker, sinks, ring, 40, n, n - 1, box, group, 1)
