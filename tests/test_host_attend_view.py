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


@pytest.mark.parametrize("sinks,ring,n,new,box,group", [(300, 300, 600, 600, 16, 1), (8, 16, 24, 24, 8, 64),
                                                        (588, 71, 579, 474, 1, 1), (700, 40, 740, 740, 128, 1),
                                                        (300, 290, 588, 588, 1, 2), (40, 20, 60, 60, 8, 40)])
def test_a_block_of_rows_at_first_positions_alone(checker, sinks, ring, n, new, box, group):
    # The ring's last positions begin at or below `sinks`, and behind the block.
    run(checker, sinks, ring, 0, n, new, box, group, 0)
    run(checker, sinks, ring, 77, n, new, box, group, 1)


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_what_rows_see(checker, seed, kind):
    run(checker, seed, 1500, kind)


@pytest.mark.parametrize("seed", [1, 2, 3])
def test_sessions_of_two_billion_tokens(checker, seed):
    # The next lap of the ring would begin beyond 2^31.
    run(checker, seed, 1500, 2)
