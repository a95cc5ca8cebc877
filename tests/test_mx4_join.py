"""What a product in 4 microscaled bits reads of a residual where several groups of waves join their sums: its own tile once, and no
row that another workgroup may be writing (the residual may be the result)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")


@pytest.fixture(scope="module")
def rows(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("join") / "mx4_join")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2510_23264_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "mx4_join.cpp"), "-o", exe], check=True)

    def run(*case):
        text = subprocess.run([exe], input="%d %d %d %d %d\n" % case, stdout=subprocess.PIPE, text=True, check=True).stdout.split()
        return [tuple(int(v) for v in pair.split(":")) for pair in text]
    return run


@pytest.mark.parametrize("tile, threads", [(32, 256), (64, 256), (64, 128)])         # the forms of several groups
@pytest.mark.parametrize("each", [4, 8])                                             # fp32, 16 bits
@pytest.mark.parametrize("left", [1, 2, 31, 32, 33, 63, 64, 65, 1000])
def test_a_tile_is_read_once_and_nothing_beside_it(rows, tile, threads, each, left):
    got = rows(tile, threads, tile, each, left)
    assert sorted(got) == [(r, c) for r in range(min(tile, left)) for c in range(0, tile, each)]


def test_the_kernel_asks_before_it_reads(rows):
    """Both the residual that is read ahead and the sums that are stored stand behind the rule the test above checks."""
    source = open(os.path.join(ROOT, "paper_2510_23264_amd", "csrc", "mx4.hip")).read()
    join = source[source.index("if constexpr (KW > 1)"):]
    join = join[:join.index("return;")]
    ahead = [line for line in join.split("\n") if "load16(" in line]
    assert len(ahead) == 1 and "mx4_in_tile(rl + r * DOWN, H, m - m0)" in ahead[0]
    assert join.index("!mx4_in_tile(rl + r * DOWN, H, m - m0)") < join.index("finish(")
