"""How the attention over a paged cache is shared out to workgroups, on the CPU: csrc/kv_plan.h compiled by itself and followed as the
workgroups follow it; and what the built kernels of the operators hold."""
import os
import random
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_23264_amd", "csrc")
FEW, MANY = (256, 4, 2, 8, 1280), (512, 4, 5, 18, 0)                 # slots, least, over, brief, enough


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    exe = str(tmp_path_factory.mktemp("plan") / "kv_plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + CSRC, os.path.join(ROOT, "tests", "host", "kv_plan.cpp"), "-o", exe], check=True)

    def run(calls, *mode):
        """For each (rule, unit, [(tiles, heads, length)]): ranges, units, the longest tile's, the longest range's, and whether all is in its place."""
        text = "".join(" ".join(map(str, c if mode else (*c[0], c[1], len(c[2]), *(v for s in c[2] for v in s)))) + "\n" for c in calls)
        out = subprocess.run([exe, *mode], input=text, stdout=subprocess.PIPE, text=True, check=True).stdout.splitlines()
        assert len(out) == len(calls)
        return [tuple(map(int, x.split())) for x in out]
    return run


def test_ranges_hold_every_unit_once(plan):
    rng = random.Random(7)

    def log_int(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))
    calls = []
    for _ in range(4000):
        rule, unit = rng.choice([FEW, MANY, (512, 4, 2, 8, 2560), (3, 1, 2, 0, 0), (7, 1, 5, 1, 100)]), rng.choice([32, 64, 128])
        heads = log_int(1, 64)
        calls.append((rule, unit, [(rng.choice([0, 1, 1, 1, log_int(1, 20)]), heads, rng.choice([0, 1, unit, log_int(1, 20000)])) for _ in range(log_int(1, 40))]))
    got = plan(calls)
    assert all(g[4] for g in got), [c for c, g in zip(calls, got) if not g[4]][:1]
    cut = [g for g in got if g[0]]
    assert 500 < len(cut) < 3900
    for wgs, units, _, most, _ in cut:
        assert most <= -(-units // wgs)                              # no range is longer than the others by more than a unit
    for (rule, *_), (wgs, units, *_) in zip(calls, got):
        assert wgs == 0 or wgs == 1 or units // wgs >= rule[1]


def test_where_tiles_are_cut(plan):
    one = [plan([(FEW, 128, [(1, 8, n)])])[0][0] for n in (0, 1, 700, 2000, 131072)]
    assert one[:3] == [0, 0, 0] and 1 < one[3] < 256 and one[4] == 256
    # as many tiles as compute units, all equal: whole; somewhat more: cut; very many: whole
    assert [plan([(FEW, 128, [(1, 8, 4096)] * n)])[0][0] for n in (32, 40, 150, 200)] == [0, 256, 256, 0]
    # one long sequence among them
    assert plan([(FEW, 128, [(1, 8, 4096)] * 200 + [(1, 8, 200000)])])[0][0] == 256
    # units that 32 bits do not count
    assert plan([(FEW, 1, [(1, 8, 2 ** 31 - 70000)])])[0][1] == 2 ** 32 - 1 and plan([(FEW, 1, [(1, 8, 2 ** 31 - 70000)])])[0][0] == 0


def test_couples_of_tiles_fit_their_units(plan):
    """A late and an early tile of a causal sequence together: never more than what the line counts for them, and at most four units and a tile's rows less."""
    rng = random.Random(8)
    calls = []
    for _ in range(20000):
        rows, group, unit = rng.choice([16, 32, 128]), rng.choice([1, 2, 3, 4, 7, 16, 33, 130]), rng.choice([32, 64, 128, 256])
        n = int(2 ** rng.uniform(0, 13))
        calls.append((n, rng.choice([n, n + int(2 ** rng.uniform(0, 30)), rng.randrange(n + 1), 0, 2 ** 31 - 70000]), rows, group, unit, rng.choice([2, 5])))
    for (n, length, rows, group, unit, over), (tiles, each, most, fewest) in zip(calls, plan(calls, "couples")):
        if tiles > 1:
            assert most <= each
            if length >= n:
                assert each - fewest <= 4 + (rows // group + 2) // unit, (n, length, rows, group, unit)


@pytest.mark.parametrize("source", ["kv_attention", "kv_cache"])
def test_kernels_keep_their_values_in_registers(tmp_path, source):
    """Spilled registers would travel through memory in the innermost loops."""
    path, llvm = os.path.join(ROOT, "paper_2510_23264_amd", "_build", source + ".o"), "/opt/rocm/llvm/bin/"
    if not os.path.exists(path) or not os.path.exists(llvm + "llvm-readelf"):
        pytest.skip("no object files or no tools to read them")
    fat, code = str(tmp_path / "fat"), str(tmp_path / "code")
    subprocess.run([llvm + "llvm-objcopy", "--dump-section", ".hip_fatbin=" + fat, path, str(tmp_path / "copy.o")], check=True)
    subprocess.run([llvm + "clang-offload-bundler", "--type=o", "--unbundle", "--input=" + fat, "--output=" + code,
                    "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"], check=True)
    notes = subprocess.run([llvm + "llvm-readelf", "--notes", code], stdout=subprocess.PIPE, text=True, check=True).stdout
    scratch = {re.search(r"\.name:\s+(\w+)", b).group(1): int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", b).group(1)) for b in notes.split("- .agpr_count:")[1:]}
    assert len(scratch) >= 7 and not any(scratch.values()), scratch
