"""Products in 4 microscaled bits at the largest sizes a call takes: every launch counts its threads in 32 bits."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MOST = (1 << 27) - 8                              # groups of 256 elements of a matrix


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_every_launch_has_fewer_than_2_to_the_32_threads(tmp_path):
    exe = str(tmp_path / "mx4_launch")
    subprocess.run(["g++", "-std=c++17", "-O1", "-ffp-contract=off", "-I" + os.path.join(ROOT, "paper_2510_23264_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "mx4_launch.cpp"), "-o", exe], check=True)
    sizes = [(m, n, k) for m in (1, 4, 5, 16, 17, 300, 70000) for k in (1, 256, 257, 4096, 1 << 24)
             for n in (1, 4096, MOST // -(-k // 256), *range((1 << 27) - 17, MOST + 1)) if n * -(-k // 256) <= MOST and m * -(-k // 256) <= MOST]
    lines = subprocess.run([exe], input="".join("%d %d %d\n" % s for s in sizes), stdout=subprocess.PIPE, text=True, check=True).stdout.split("\n")
    got = {s: tuple(int(v) for v in line.split()) for s, line in zip(sizes, lines)}
    assert len(got) > 150 and all(threads < 1 << 32 for _, threads in got.values())
    assert got[(16, (1 << 27) - 16, 256)] == (-1, (1 << 32) - 512)          # the last size the kernel of few rows counts
    assert all(got[(m, n, 256)][0] >= 0 for m in (1, 16) for n in range((1 << 27) - 15, MOST + 1))


@pytest.mark.gpu
def test_few_rows_by_the_most_columns():
    """2^27 - 15 and more rows of weights (17 GB): exact sums (scales of 1), the first, middle and last against calls on them alone."""
    import torch
    import paper_2510_23264_amd as P
    torch.manual_seed(2)
    a = P.Mx4(torch.randint(0, 256, (2, 128), device="cuda", dtype=torch.uint8), torch.full((2, 8), 127, device="cuda", dtype=torch.uint8), 256)
    codes = torch.randint(0, 256, (MOST, 128), device="cuda", dtype=torch.uint8)
    scales = torch.full((MOST, 8), 127, device="cuda", dtype=torch.uint8)
    for n in ((1 << 27) - 16, (1 << 27) - 15, MOST):
        out = P.mx4_gemm(a, P.Mx4(codes[:n], scales[:n], 256))
        for lo in (0, (1 << 25) - 7, (1 << 26) + 1, n - 40):
            part = P.Mx4(codes[lo:lo + 40], scales[lo:lo + 40], 256)
            assert torch.equal(out[:, lo:lo + 40], P.mx4_gemm(a, part)), (n, lo)
        del out
