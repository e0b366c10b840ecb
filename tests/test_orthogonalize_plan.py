"""The rule that chooses the kernels of trivance_orthogonalize, on the CPU: every form that it takes for any sizes
is one that the GPU tests run, and what a form launches fits its indexes."""

import math
import os
import random
import subprocess

import pytest

pytest.importorskip("torch")

import orthogonalize_util as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_17254_amd", "csrc")


@pytest.fixture(scope="module")
def form_of(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "orthogonalize_plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I", CSRC,
                    os.path.join(ROOT, "tests", "c", "orthogonalize_plan.cpp"), "-o", exe], check=True)

    def forms(sizes):
        lines = "\n".join("%d %d %d" % s for s in sizes)
        out = subprocess.run([exe], input=lines, capture_output=True, text=True, check=True, timeout=300).stdout
        got = [line.split(" ", 3) for line in out.splitlines()]
        assert [tuple(map(int, g[:3])) for g in got] == list(sizes)
        return [g[3] for g in got]

    return forms


def test_listed_sizes_take_their_forms(form_of):
    assert form_of(ref.FORMS.values()) == list(ref.FORMS)


def test_no_size_takes_another_form(form_of):
    rng = random.Random(1)
    sizes = [(1, m, n) for m in range(1, 200, 9) for n in (m, 256, 257, 8192, 8193, 65536)]
    sizes += [(b, 64 * i, 64 * j) for b in (1, 3, 8) for i in range(1, 41) for j in range(i, 121, 3)]
    for _ in range(60000):
        m = int(math.exp(rng.uniform(0, math.log(65536))))
        n = int(math.exp(rng.uniform(math.log(m), math.log(65536))))
        sizes.append((rng.choice([1, 1, 1, 2, 3, 4, 8, 16, 64, 300, 65535]), m, n))
    # what fits a GPU's memory: 16 bytes a value of X and more
    sizes = [s for s in sizes if s[0] * max(s[1], 64) * max(s[2], 64) < 1 << 34]
    assert set(form_of(sizes)) <= set(ref.FORMS)
