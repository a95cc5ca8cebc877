"""Appending to a paged cache and keeping a path of a drafted tree, on the device."""
import numpy as np
import pytest
import torch

from plain_kv import ORDERS, Case, attend, check, random_tree, seen_of

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def P():
    import paper_2510_23264_amd as p
    return p


def written(case, keys, values, k, v):
    """The cache after the new tokens' rows are put one by one."""
    keys, values = keys.clone(), values.clone()
    for b, n in enumerate(case.new):
        for i in range(n):
            row, t = case.lengths[b] - n + i, int(case.starts[b]) + i
            if row >= 0:
                keys[case.table[b][row // case.page], :, row % case.page] = k[t]
                values[case.table[b][row // case.page], :, row % case.page] = v[t]
    return keys, values


def same(a, b):
    return torch.equal(torch.nan_to_num(a.cpu().float(), 77.0), torch.nan_to_num(b.cpu().float(), 77.0))


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("new, lengths, heads, group, d, rot, page", [
    ((1,), (1,), 1, 1, 8, 2, 1), ((1, 1, 1, 1), (9, 100, 17, 33), 8, 4, 128, 128, 16), ((5, 0, 30), (5, 9, 90), 2, 3, 80, 20, 24), ((3, 2), (40, 30), 1, 7, 64, 16, 7),
    ((70, 1300), (70, 2000), 2, 1, 32, 32, 64), ((2500,), (2500,), 1, 2, 96, 50, 100), ((9,), (50,), 3, 1, 256, 256, 16), ((33,), (64,), 2, 2, 16, 10, 5)])
def test_rows_are_what_rotary_gives(P, dtype, layout, new, lengths, heads, group, d, rot, page):
    """Keys and queries bit for bit as pahq_rotary turns them, values as they are, everything else in the cache untouched."""
    for order, part in (("heads", False), ("slots", True), ("joined", True)):
        case = Case(new, lengths, heads, group, d, page, dtype, order=order)
        cache, batch, q = case.device(P)
        rows = torch.randn(case.tokens, heads * (group + 2) * d + 3, device="cuda").to(dtype)
        if part:                                                       # parts of one projection's rows, at an odd start
            at = rows[:, 1:1 + heads * (group + 2) * d].view(case.tokens, heads * (group + 2), d)
            q, k, v = at.split([heads * group, heads, heads], dim=1)
        else:
            k, v = torch.randn(2, case.tokens, heads, d, device="cuda").to(dtype)
        table = P.rotary_table(rot, theta=500.0)
        positions = torch.randint(-5, 1 << 20, (case.tokens,), device="cuda")
        want_q, want_k = (P.rotary(x, positions, table, layout=layout, magnitude=1.25) for x in (q, k))
        keys, values = written(case, case.keys, case.values, want_k.cpu(), v.cpu())
        before = rows.clone()
        got = P.kv_append(cache, batch, k, v, positions=positions, table=table, layout=layout, magnitude=1.25, q=q)
        assert torch.equal(got, want_q) and same(cache.keys, keys) and same(cache.values, values) and torch.equal(rows, before)
        assert P.kv_append(cache, batch, k, v, positions=positions, table=table, layout=layout, magnitude=1.25, q=q, out=q) is not None
        assert torch.equal(q, want_q)
        # positions of their own: the tokens' rows; and nothing turned
        where = torch.cat([torch.arange(n) + length - n for n, length in zip(new, lengths)]).cuda()
        keys, values = written(case, case.keys, case.values, P.rotary(k, where, table, layout=layout).cpu(), v.cpu())
        assert P.kv_append(cache, batch, k, v, table=table, layout=layout) is None
        assert same(cache.keys, keys) and same(cache.values, values)
        assert torch.equal(P.kv_append(cache, batch, k, v, q=q), q)
        assert same(cache.keys, written(case, case.keys, case.values, k.cpu(), v.cpu())[0])


def test_tokens_without_a_place(P):
    """Padding in front and behind, rows that would be negative or behind the list, pages that are none: not written; queries of tokens that
    belong to a sequence are turned all the same."""
    for dtype in DTYPES:
        case = Case((3, 4, 2), (40, 20, 2), 2, 2, 64, 16, dtype, fill=0.0)
        cache, batch, q = case.device(P)
        k, v = torch.randn(2, 14, 2, 64, device="cuda").to(dtype)
        q = torch.randn(14, 4, 64, device="cuda").to(dtype)
        shifted = P.KvBatch(batch.starts + 2, batch.lengths.clone(), batch.pages.clone())
        shifted.lengths[0] = 2                                          # its first token has no row
        shifted.pages[1, 1] = 1 << 20
        shifted.lengths[2] = 1000                                       # clipped to the list's room, of which only one page is real
        table = P.rotary_table(64)
        out = torch.full_like(q, 3.0)
        keys, values = cache.keys.clone(), cache.values.clone()
        P.kv_append(cache, shifted, k, v, table=table, q=q, out=out)
        assert (out[:2] == 3).all() and (out[11:] == 3).all()
        where = torch.tensor([0, 0, -1, 0, 1, 16, 17, 18, 19, 46, 47, 0, 0, 0], device="cuda")
        assert torch.equal(out[2:11], P.rotary(q, where, table)[2:11])
        turned = P.rotary(k, where, table)
        for t, row in ((3, 0), (4, 1)):
            keys[case.table[0][0], :, row], values[case.table[0][0], :, row] = turned[t], v[t]
        assert torch.equal(cache.keys, keys) and torch.equal(cache.values, values)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_a_list_that_is_too_short_costs_no_row(P, dtype):
    """A sequence that has outgrown its list of pages: nothing of it is written or moved, and the rows that it has stay."""
    for length in (33, 40, 1000, 2 ** 31 - 1):
        case = Case((3, 2), (32, 20), 2, 2, 64, 16, dtype)
        cache, batch, q = case.device(P)
        k, v = torch.randn(2, 5, 2, 64, device="cuda").to(dtype)
        batch.lengths[0] = length
        keys, values = case.keys.clone(), case.values.clone()
        for i, row in enumerate((18, 19)):                              # the other sequence's rows
            keys[case.table[1][row // 16], :, row % 16], values[case.table[1][row // 16], :, row % 16] = k[3 + i].cpu(), v[3 + i].cpu()
        P.kv_append(cache, batch, k, v)
        assert same(cache.keys, keys) and same(cache.values, values)
        after = P.kv_keep(cache, batch, torch.tensor([[1, 2], [1, -1]], dtype=torch.int32, device="cuda"))
        assert after[1] == 19
        for rows in (keys, values):
            rows[case.table[1][18 // 16], :, 18 % 16] = rows[case.table[1][19 // 16], :, 19 % 16]
        assert same(cache.keys, keys) and same(cache.values, values)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("heads, d, page, order", [(1, 8, 1, "heads"), (2, 128, 16, "joined"), (3, 256, 7, "slots"), (12, 64, 32, "outer slots"), (5, 80, 24, "heads")])
def test_keep_moves_a_path(P, dtype, heads, d, page, order):
    """Against moving all rows at once: paths of every kind, also ones that end early because they do not grow or leave the tree."""
    new, lengths = (26, 64, 1, 9, 0, 130), (100, 64, 30, 9, 12, 131)
    paths = torch.tensor([[0, 3, 7, 25, -1, -1, -1], [1, 2, 3, 4, 5, 6, 7], [0, -1, 5, -1, -1, -1, -1], [2, 4, 4, 6, 8, -1, -1], [0, 1, 2, 3, 4, 5, 6],
                          [0, 5, 64, 127, 129, 130, 131]], dtype=torch.int32)
    stay = [4, 7, 1, 2, 0, 5]
    case = Case(new, lengths, heads, 1, d, page, dtype, order=order)
    cache, batch, _ = case.device(P)
    keys, values = case.keys.clone(), case.values.clone()
    for b, n in enumerate(stay):
        base = lengths[b] - new[b]
        for i in range(n):
            x, y = base + int(paths[b, i]), base + i
            for to, of in ((keys, case.keys), (values, case.values)):
                to[case.table[b][y // page], :, y % page] = of[case.table[b][x // page], :, x % page]
    got = P.kv_keep(cache, batch, paths.cuda())
    assert got.tolist() == [length - n + s for length, n, s in zip(lengths, new, stay)] and got.dtype == torch.int32
    assert same(cache.keys, keys) and same(cache.values, values)


def test_keep_of_long_paths(P):
    """Paths longer than a workgroup and a wave hold at a time: every second token, all tokens, all but the first."""
    for dtype in DTYPES:
        case = Case((600, 200, 200), (700, 200, 333), 2, 1, 256, 48, dtype)
        cache, batch, _ = case.device(P)
        paths = torch.full((3, 320), -1, dtype=torch.int32)
        paths[0, :300] = torch.arange(0, 600, 2)
        paths[1, :200] = torch.arange(200)
        paths[2, :199] = torch.arange(1, 200)
        out = torch.empty(3, dtype=torch.int32, device="cuda")
        rows = [case.rows(case.keys, b) for b in range(3)]
        assert P.kv_keep(cache, batch, paths.cuda(), out=out) is not None and out.tolist() == [400, 200, 332]
        for b, (base, n) in enumerate(((100, 300), (0, 200), (133, 199))):
            got = case.rows(cache.keys.cpu(), b)
            want = rows[b].clone()
            want[base:base + n] = rows[b][base + paths[b, :n].long()]
            assert torch.equal(got, want)
        assert P.kv_keep(cache, batch, paths[:, :0].cuda()).tolist() == [100, 0, 133]


def test_keep_leaves_rows_that_cannot_be_read(P):
    case = Case((40,), (40,), 2, 1, 64, 16, torch.bfloat16)
    cache, batch, _ = case.device(P)
    batch.pages[0, 1] = -3
    before = cache.keys.clone()
    assert P.kv_keep(cache, batch, torch.tensor([[1, 17, 33, 34]], dtype=torch.int32, device="cuda")).tolist() == [4]
    before[case.table[0][0], :, 0] = before[case.table[0][0], :, 1]
    before[case.table[0][0], :, 2:4] = before[case.table[0][2], :, 1:3]
    assert same(cache.keys, before)


def test_a_drafted_tree_end_to_end(P):
    """A program's loop: a prompt, then drafts of trees that are appended, attended and cut back to a path; every step's attention is that of the
    plain sequence along each node's ancestors, and at the end the cache holds what appending the accepted tokens alone leaves."""
    torch.manual_seed(2)
    heads, group, d, page, dtype = 2, 3, 64, 16, torch.float32
    table = P.rotary_table(32, theta=1000.0)
    cache = P.KvCache.empty(40, page, heads, d, dtype)
    plain = P.KvCache.empty(40, page, heads, d, dtype)
    pages = torch.randperm(40, device="cuda").to(torch.int32).view(2, 20)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")      # noqa: E731
    prompt = [37, 5]
    q, k, v = torch.randn(42, 10, d, device="cuda").split([6, 2, 2], dim=1)
    batch = P.KvBatch(i32(0, 37, 42), i32(*prompt), pages)
    for c in (cache, plain):
        turned = P.kv_append(c, batch, k, v, table=table, q=q)
    lengths = torch.tensor(prompt)
    g = torch.Generator().manual_seed(1)
    for step in range(4):
        n = 20 + 30 * (step % 2)
        parents = [random_tree(n, g) for _ in range(2)]
        depth = [[0] * n for _ in range(2)]
        for b in range(2):
            for i in range(1, n):
                depth[b][i] = depth[b][parents[b][i]] + 1
        positions = torch.cat([lengths[b] + torch.tensor(depth[b]) for b in range(2)]).cuda()
        q, k, v = torch.randn(2 * n, 10, d, device="cuda").split([6, 2, 2], dim=1)
        batch = P.KvBatch(i32(0, n, 2 * n), (lengths + n).to(torch.int32).cuda(), pages)
        turned = P.kv_append(cache, batch, k, v, positions=positions, table=table, q=q)
        tree = torch.cat([P.tree_bits(p) for p in parents])
        got = P.kv_attention(turned, cache, batch, tree=tree)
        paths = torch.full((2, 6), -1, dtype=torch.int32)
        for b in range(2):
            path = [n - 1]
            while parents[b][path[0]] >= 0:
                path.insert(0, parents[b][path[0]])
            path = path[:6]
            paths[b, :len(path)] = torch.tensor(path)
            # the path alone, appended to the plain cache one after the other, each attending causally
            one = P.KvBatch(i32(0, len(path)), i32(int(lengths[b]) + len(path)), pages[b:b + 1])
            at = torch.tensor(path, device="cuda") + b * n
            alone = P.kv_append(plain, one, k[at], v[at], table=table, q=q[at])
            want = P.kv_attention(alone, plain, one)
            assert torch.equal(turned[at], alone)
            assert (got[at] - want).abs().max() <= 1e-5 * want.abs().max()      # the same sums over other tiles, in fp32
        lengths = P.kv_keep(cache, batch, paths.cuda()).cpu().long()
        for b in range(2):
            for c, o in ((cache.keys, plain.keys), (cache.values, plain.values)):
                a, w = (t[pages[b].long()].transpose(1, 2).reshape(-1, heads, d)[:lengths[b]] for t in (c, o))
                assert torch.equal(a, w)


def test_a_layer_of_operators(P):
    """Rows in 4 bits, their product, append with rotation, attention, rows in 4 bits, the product on the residual: as a program calls them,
    against the same steps in 64 bits on the values the codes stand for."""
    torch.manual_seed(4)
    heads, group, d, width = 2, 4, 64, 512
    w_in = P.mx4_quantize(torch.randn(width, (heads * (group + 2)) * d, device="cuda") * 0.04, by="columns")
    w_out = P.mx4_quantize(torch.randn(heads * group * d, width, device="cuda") * 0.04, by="columns")
    case = Case((33, 1), (60, 130), heads, group, d, 16, torch.float32)
    cache, batch, _ = case.device(P)
    x = torch.randn(34, width, device="cuda")
    table = P.rotary_table(d)
    qkv = P.mx4_gemm(P.mx4_quantize(x), w_in)
    q, k, v = qkv.view(34, heads * (group + 2), d).split([heads * group, heads, heads], dim=1)
    turned = P.kv_append(cache, batch, k, v, table=table, q=q, out=q)
    o = P.kv_attention(turned, cache, batch)
    y = P.mx4_gemm(P.mx4_quantize(o.view(34, -1)), w_out, residual=x)
    case.keys, case.values, case.q = cache.keys.cpu(), cache.values.cpu(), turned.cpu()
    check(o, *attend(case))
    want = P.mx4_dequantize(P.mx4_quantize(o.view(34, -1))).double() @ P.mx4_dequantize(w_out).double().t().contiguous() + x.double()
    assert (y.double() - want).abs().max() <= 1e-5 * want.abs().max()


def test_the_first_call_is_a_captured_one():
    import os
    import subprocess
    import sys
    code = """
import torch
import paper_2510_23264_amd as P
cache = P.KvCache.empty(40, 16, 2, 64)
cache.keys.normal_(); cache.values.normal_()
i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
batch = P.KvBatch(i32(0, 1, 40), i32(300, 90), torch.arange(40, device="cuda").to(torch.int32).view(2, 20))
q, k, v = torch.randn(40, 12, 64, device="cuda").to(torch.bfloat16).split([8, 2, 2], dim=1)
paths = i32(0, -1, 0, 5).view(2, 2)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    P.kv_append(cache, batch, k, v, q=q)
    got = P.kv_attention(q, cache, batch)
    after = P.kv_keep(cache, batch, paths)
for _ in range(3):
    q.normal_()
    graph.replay()
    torch.cuda.synchronize()
    P.kv_append(cache, batch, k, v)
    assert torch.equal(got, P.kv_attention(q, cache, batch)) and after.tolist() == [300, 53]
print("replayed")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    got = subprocess.run([sys.executable, "-c", code], cwd=root, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=100)
    assert got.returncode == 0 and "replayed" in got.stdout, got.stdout
