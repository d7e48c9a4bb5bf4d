"""CPU: the warps that fill a ring together give up together
(tests/host/rounds_check.cpp over csrc/pcs_attend_rounds.h, built here with
g++), and wait for what they sent (tests/host/rings_check.cpp)."""
import os
import shutil
import subprocess

import pytest

from paper_2607_21686_gb300 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_warps_give_up_together(tmp_path):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no g++")
    exe = tmp_path / "rounds_check"
    subprocess.run([gxx, "-O1", "-std=c++17", "-pthread", "-I", build.CSRC,
                    os.path.join(ROOT, "tests", "host", "rounds_check.cpp"), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr


def test_copies_are_waited_for(tmp_path):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no g++")
    exe = tmp_path / "rings_check"
    subprocess.run([gxx, "-O1", "-std=c++17", "-I", build.CSRC,
                    os.path.join(ROOT, "tests", "host", "rings_check.cpp"), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr
