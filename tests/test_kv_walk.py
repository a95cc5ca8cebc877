"""Who does what of an attention over a paged cache, and every address of it, on the CPU: csrc/kv_plan.h and csrc/kv_address.h, from which the
kernels take both, compiled by themselves and followed lane by lane (host/kv_walk.cpp).  Every tile's rows are taken once, what the join reads
was written, LDS holds what the products read there, and no address leaves the cache, the lists, the operands' rows, LDS or the workspace."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HUGE = 2 ** 31 - 1


@pytest.fixture(scope="module")
def follow(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    exe = str(tmp_path_factory.mktemp("walk") / "kv_walk")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I" + os.path.join(ROOT, "paper_2510_23264_amd", "csrc"), os.path.join(ROOT, "tests", "host", "kv_walk.cpp"), "-o", exe],
                   check=True)

    def run(mode, lines=()):
        out = subprocess.run([exe, mode], input="".join(" ".join(map(str, x)) + "\n" for x in lines), stdout=subprocess.PIPE, text=True, check=True).stdout.splitlines()
        assert len(out) == (len(lines) if mode != "stages" else 6)
        bad = [(x, y) for x, y in zip(lines or out, out) if not y[0].isdigit()]
        assert not bad, (len(bad), [(str(x)[:300], y) for x, y in bad[:3]])
        return [tuple(map(int, y.split())) for y in out]
    return run


def test_the_quotient_of_a_page_size_is_the_division(follow):
    rng = random.Random(1)
    sizes = [1, 2, 3, 5, 7, 16, 24, 48, 100, 255, 256, 257, 65535, 65537, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, HUGE - 1, HUGE]
    follow("quotient", [(p,) for p in sizes + [rng.randrange(1, HUGE) for _ in range(2000)] + [int(2 ** rng.uniform(0, 31)) for _ in range(2000)]])


def test_bits_of_what_a_query_sees(follow):
    rng = random.Random(2)
    lines = []
    for _ in range(600):
        base, n, words = rng.choice([0, 1, 63, 64, 65, 1000, -3, -64, -100]), rng.choice([1, 2, 30, 63, 64, 65, 100, 130]), rng.choice([1, 1, 2, 3])
        k0 = rng.choice([0, 16, 32, 48, 64, 128, max(0, base // 16 * 16), max(0, (base + n) // 32 * 32)])
        lines.append((words, base, n, k0, rng.choice([max(0, base + n), k0 + rng.randrange(70)])))
    follow("seen", lines)


def test_what_is_brought_to_lds_is_what_the_products_read(follow):
    follow("stages")


def call(eb, causal, new, lengths, heads, group, d, page_size, layout=0, spare=3, width=None, starts=None, tokens=None, sane=1):
    own = [0]
    for n in new:
        own.append(own[-1] + n)
    width = max([-(-x // page_size) for x in lengths] + [1]) if width is None else width
    pages = min(sum(-(-x // page_size) for x in lengths if x > 0) + spare, HUGE)
    starts = own if starts is None else starts
    return (eb, causal, own[-1] if tokens is None else tokens, len(new), heads, group, d, page_size, max(pages, 1), width, layout, sane, *starts, *lengths)


def test_calls_that_the_device_runs(follow):
    """Shapes of the tests on the device, those among them on which a kernel that is gone faulted, in both types and every layout of the cache; lists of pages
    as long as the sequences, and much longer, with which more of them are cut."""
    shapes = [((1,), (1,), 1, 1, 8, 1), ((1, 1, 1), (31, 32, 33), 2, 4, 64, 16), ((1, 1), (65, 300), 1, 7, 128, 24), ((1,), (129,), 3, 16, 256, 64), ((5,), (5,), 2, 3, 80, 8),
              ((2, 9, 0, 1), (64, 9, 40, 1), 2, 4, 32, 16), ((70, 3), (70, 131), 1, 5, 40, 7), ((130,), (259,), 1, 1, 192, 16), ((257, 20), (300, 300), 1, 2, 64, 64),
              ((40,), (40,), 1, 12, 72, 256), ((129,), (129,), 2, 1, 256, 48), ((1,), (1000,), 1, 48, 128, 1), ((100,), (100,), 1, 3, 224, 64), ((100,), (300,), 1, 3, 224, 64),
              ((100,), (300,), 1, 3, 256, 64), ((97,), (97,), 1, 3, 192, 16), ((44,), (100,), 1, 1, 256, 64), ((97, 36), (300, 36), 2, 1, 64, 16), ((1,), (9001,), 1, 4, 64, 16),
              ((1, 1, 1, 1), (3, 7000, 64, 1500), 2, 2, 128, 64), ((100,), (4100,), 1, 2, 128, 16), ((6,), (3000,), 2, 4, 256, 32), ((1, 300, 2), (4000, 900, 1), 1, 1, 64, 100),
              ((64,) * 8, (100, 8000, 900, 64, 3000, 70, 500, 5000), 8, 4, 128, 16), ((1500, 20, 700, 33), (1500, 4000, 2100, 33), 12, 1, 64, 16), ((8192,), (8192,), 8, 4, 128, 64),
              ((5,), (3,), 2, 1, 64, 16), ((0, 0, 2), (0, 0, 2), 1, 1, 128, 32), ((333, 100), (2100, 400), 5, 3, 80, 24), ((1,), (131072,), 8, 4, 128, 64)]
    got = follow("walk", [call(eb, causal, *s, layout=layout, width=w) for s in shapes for eb in (2, 4) for causal in (1, 0) for layout in (0, 1, 2)
                          for w in (None, -(-max(s[1]) // s[5]) + 3000)])
    assert {16, 32, 128} <= {g[0] for g in got} and sum(g[1] > 0 for g in got) > 150 and sum(g[1] == 0 for g in got) > 150


def test_calls_at_random(follow):
    rng = random.Random(3)

    def log_int(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))
    lines = []
    for _ in range(900):
        batch = log_int(1, 300)
        kind = rng.choice(["token", "few", "many", "mixed"])
        new = [1 if kind == "token" else log_int(1, 12) if kind == "few" else log_int(1, 3000 if batch < 5 else 300) if kind == "many" else rng.choice([0, 1, 1, 1, log_int(1, 500)])
               for _ in range(batch)]
        far = rng.choice([50, 1000, 30000])
        lengths = [n + rng.choice([0, log_int(1, far), log_int(1, far)]) for n in new]
        page = rng.choice([1, 5, 8, 16, 24, 32, 64, 100, 256])
        width = None if rng.random() < 0.5 else -(-max(lengths) // page) + log_int(1, 3000 if batch < 50 else 100)
        lines.append(call(rng.choice([2, 4]), rng.choice([1, 0]), new, lengths, rng.choice([1, 2, 3, 8, 12]), rng.choice([1, 1, 2, 4, 7, 33]), 8 * rng.randint(1, 32), page,
                          layout=rng.randrange(3), width=width))
    got = follow("walk", [x for x in lines if x[2]])
    assert min(sum(g[0] == rows and (g[1] > 0) == cut for g in got) for rows in (16, 32, 128) for cut in (True, False)) > 15


def test_batches_whose_numbers_make_no_sense_stay_in_range(follow):
    rng = random.Random(4)
    lines = []
    for _ in range(700):
        batch, tokens = rng.choice([1, 2, 3, 5, 40, 100]), rng.choice([1, 3, 40, 44, 500, 3000])

        def start():
            return rng.choice([0, tokens, rng.randrange(tokens + 1), rng.randrange(tokens + 1), -5, tokens + 100, HUGE, -2 ** 31])
        page, width = rng.choice([1, 16, 24, 64]), rng.choice([1, 4, 30, 400, 3000])
        lengths = [rng.choice([0, -1, -2 ** 31, HUGE, rng.randrange(width * page + 1), width * page + 7, rng.randrange(100)]) for _ in range(batch)]
        lines.append(call(rng.choice([2, 4]), rng.choice([1, 0]), [1] * batch, [5] * batch, rng.choice([1, 2, 8]), rng.choice([1, 3, 4]), rng.choice([64, 128, 224, 256]), page,
                          layout=rng.randrange(3), width=width, starts=[start() for _ in range(batch + 1)], tokens=tokens, sane=0)[:-batch] + tuple(lengths))
    follow("walk", lines)


def test_sequences_as_long_as_rows_are_counted(follow):
    """Lists that have room for 2^31 - 65536 rows and more (of pages of 2^20 rows): one token, a few, and a tile's worth."""
    page = 1 << 20
    follow("walk", [call(eb, causal, (n,), (length,), 1, 1, d, page, width=2048) for eb in (2, 4) for causal in (0, 1) for d in (64, 256) for n in (1, 20, 200)
                    for length in (HUGE - 65536, HUGE, 2 ** 30 + 1)])
