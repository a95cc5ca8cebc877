"""The rule of the products in 4 microscaled bits, on the CPU: csrc/mx4_rules.h compiled by itself, against the copy the GPU
tests use and against what its comments state."""
import os
import random
import shutil
import subprocess
import sys

import pytest

sys.path.insert(0, os.path.dirname(__file__))
import mx4_rules as R                              # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")


@pytest.fixture(scope="module")
def pick(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("rules") / "mx4_rules")
    subprocess.run(["g++", "-std=c++17", "-O1", "-ffp-contract=off", "-I" + os.path.join(ROOT, "paper_2510_23264_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "mx4_rules.cpp"), "-o", exe], check=True)

    def run(sizes):
        text = "".join("%d %d %d\n" % q for q in sizes)
        out = subprocess.run([exe], input=text, stdout=subprocess.PIPE, text=True, check=True).stdout.split()
        assert len(out) == len(sizes)
        return [int(v) for v in out]
    return run


def test_the_copy_agrees(pick):
    """The library computes in binary32: where two estimates are closer than that, either may be taken."""
    rng = random.Random(5)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))       # noqa: E731
    sizes = [(log(1, 40000), log(1, 60000), log(1, 20000)) for _ in range(20000)] + [(1 << 31, 1 << 31, 1 << 24), (1, 1, 1)]
    for size, got in zip(sizes, pick(sizes)):
        want = R.form(*size)
        if got != want:
            slabs = -(-size[2] // 256)
            a, b = R.estimate(R.FORMS[got], size[0], size[1], slabs), R.estimate(R.FORMS[want], size[0], size[1], slabs)
            assert min(got, want) >= 0 and abs(a - b) <= 1e-5 * a, size


def test_the_sizes_its_comments_name(pick):
    assert pick([(1, 4096, 4096), (1, 1024, 16000), (1, 11008, 4096), (16, 11008, 4096), (11, 31513, 9086), (100, 2304, 768), (256, 4096, 4096), (800, 2304, 768),
                 (2048, 4096, 4096), (8192, 4096, 11008)]) == \
        [R.FEW, R.FEW, R.FEW, R.T32, R.T32, R.T32, R.T64_FOUR, R.T64_TWO, R.T128, R.T256]
