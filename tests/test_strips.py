"""The loops over strips of slots and tokens, on the CPU: tests/c/strips.cpp runs them with g++ up to the largest
numbers that the calls take."""

import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_17254_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not found")
def test_strips_end_at_the_largest_int(tmp_path):
    exe = str(tmp_path / "strips")
    subprocess.run(["g++", "-std=c++17", "-O1", "-ftrapv", "-Wall", "-Wextra", "-Werror", "-I", CSRC,
                    os.path.join(ROOT, "tests", "c", "strips.cpp"), "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0, res.stdout + res.stderr
    assert "strips ok" in res.stdout


@pytest.mark.parametrize("name", ["embedding.hip", "experts.hip"])
def test_kernels_count_by_strips(name):
    """No kernel counts slots or tokens up by whole strips in an int, which may go beyond the largest one."""
    with open(os.path.join(CSRC, name)) as f:
        assert not re.findall(r"for \(int \w+ = [^;]*;[^;]*; \w+ \+= [KL]\)", f.read())
