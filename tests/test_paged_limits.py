"""The paged cache at the ends of its ranges, on the CPU: the headers are compiled by themselves (paged_limits_check.cpp)."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2604_21215_amd", "csrc")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("paged_limits") / "check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, os.path.join(HERE, "paged_limits_check.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("check", ["codes", "launches", "overlaps"])
def test_paged_limits(program, check):
    r = subprocess.run([program, check], stdout=subprocess.PIPE, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
