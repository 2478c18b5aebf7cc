"""The MX FP4 products' tiles on the host (no GPU): tests/native/mx4_form_check.cpp
compiles csrc/mx4_form.h for the host."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_00993_amd", "csrc")


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ not found")
    exe = str(tmp_path_factory.mktemp("mx4_form") / "mx4_form_check")
    cmd = [cxx, "-O1", "-std=c++17", "-Wall", f"-I{CSRC}", os.path.join(ROOT, "tests", "native", "mx4_form_check.cpp"),
           "-o", exe]
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, f"build failed:\n{' '.join(cmd)}\n{p.stdout}"
    return exe


def test_lane_offsets_fit(check):
    r = subprocess.run([check], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout[:2000]
