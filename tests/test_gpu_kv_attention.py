"""Attention over a paged cache on the device against the definition in 64 bits.  Memory that is no sequence's is NaN, so every case
also shows that nothing is taken from there."""
import numpy as np
import pytest
import torch

from plain_kv import ORDERS, Case, attend, check, random_tree

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def P():
    import paper_2510_23264_amd as p
    return p


def run(P, case, tree=None, **how):
    cache, batch, q = case.device(P)
    return P.kv_attention(q, cache, batch, tree=None if tree is None else tree.cuda(), **how)


def trees(case, P, sizes=None):
    """Masks of a random tree for each sequence, of as many words."""
    rows = []
    words = max(1, -(-max(case.new) // 64))
    for n in case.new:
        bits = P.tree_bits(random_tree(n, case.g), device="cpu") if n else torch.zeros(0, words, dtype=torch.int64)
        rows.append(torch.nn.functional.pad(bits, (0, words - bits.shape[1])))
    return torch.cat(rows)


# lengths around tiles, waves and pages; one token, a few, more than a tile; heads of every width the kernels pad to; groups that do not divide a tile
@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("new, lengths, heads, group, d, page", [
    ((1,), (1,), 1, 1, 8, 1), ((1,), (17,), 2, 1, 16, 16), ((1, 1, 1), (31, 32, 33), 2, 4, 64, 16), ((1, 1), (65, 300), 1, 7, 128, 24),
    ((1,), (129,), 3, 16, 256, 64), ((1, 1), (5, 700), 1, 33, 96, 100), ((5,), (5,), 2, 3, 80, 8), ((2, 9, 0, 1), (64, 9, 40, 1), 2, 4, 32, 16),
    ((33, 1), (33, 64), 1, 1, 64, 32), ((64,), (200,), 2, 2, 128, 16), ((70, 3), (70, 131), 1, 5, 40, 7), ((130,), (259,), 1, 1, 192, 16),
    ((257, 20), (300, 300), 1, 2, 64, 64), ((40,), (40,), 1, 12, 72, 256), ((129,), (129,), 2, 1, 256, 48), ((1,), (1000,), 1, 48, 128, 1),
    # a wave of which some rows are queries and the rest is nobody's
    ((100,), (100,), 1, 3, 224, 64), ((100,), (300,), 1, 3, 256, 64), ((97,), (97,), 1, 3, 192, 16), ((44,), (100,), 1, 1, 256, 64), ((44,), (100,), 1, 1, 128, 64),
    ((97, 36), (300, 36), 2, 1, 64, 16)])
def test_against_the_definition(P, dtype, new, lengths, heads, group, d, page):
    case = Case(new, lengths, heads, group, d, page, dtype, seed=sum(lengths) + d)
    want, lim = attend(case)
    got = run(P, case)
    check(got, want, lim)
    assert torch.equal(got, run(P, case))
    if max(new) > 1:
        tree = trees(case, P)
        check(run(P, case, tree), *attend(case, tree))


# long contexts: split over workgroups and joined, sequences of very different length, many and one, a few rows and a tile of them
@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("new, lengths, heads, group, d, page", [
    ((1,), (9001,), 1, 4, 64, 16), ((1, 1, 1, 1), (3, 7000, 64, 1500), 2, 2, 128, 64), ((1,) * 70, tuple(range(1, 1401, 20)), 1, 1, 64, 16),
    ((20, 1, 4), (5000, 2500, 90), 1, 3, 64, 24), ((100,), (4100,), 1, 2, 128, 16), ((6,), (3000,), 2, 4, 256, 32), ((1, 300, 2), (4000, 900, 1), 1, 1, 64, 100)])
def test_long_contexts(P, dtype, new, lengths, heads, group, d, page):
    case = Case(new, lengths, heads, group, d, page, dtype, seed=sum(lengths), spread=1.5)
    check(run(P, case), *attend(case))
    if max(new) > 1:
        tree = trees(case, P)
        check(run(P, case, tree), *attend(case, tree))


@pytest.mark.parametrize("order", list(ORDERS) + ["joined"])
@pytest.mark.parametrize("new, lengths", [((1, 1), (50, 130)), ((40, 3), (77, 130))])
def test_orders_of_the_cache_in_memory(P, order, new, lengths):
    for dtype in DTYPES:
        case = Case(new, lengths, 3, 2, 64, 16, dtype, order=order)
        check(run(P, case), *attend(case))


def test_strides_of_queries_and_results(P):
    """Queries inside rows of a projection at an odd start, heads outside of tokens; results in place, in other columns, behind and in front of
    rows that stay as they were."""
    for dtype in DTYPES:
        for new, lengths in (((1, 1), (50, 130)), ((40, 3), (77, 130))):
            case = Case(new, lengths, 2, 2, 64, 16, dtype, seed=3)
            cache, batch, q = case.device(P)
            n = case.tokens
            want = P.kv_attention(q, cache, batch)
            rows = torch.randn(n, 1 + 2 * 4 * 64, device="cuda").to(dtype)
            x, y = rows[:, 1:257].view(n, 4, 64), rows[:, 257:].view(n, 4, 64)
            x.copy_(q)
            assert torch.equal(P.kv_attention(x, cache, batch), want)
            assert P.kv_attention(x, cache, batch, out=y) is not None and torch.equal(y, want) and torch.equal(x, q)
            P.kv_attention(x, cache, batch, out=x)
            assert torch.equal(x, want)
            planes = torch.empty(4, n, 64, dtype=dtype, device="cuda").transpose(0, 1)
            assert torch.equal(P.kv_attention(planes.copy_(q), cache, batch), want)
            assert torch.equal(P.kv_attention(q, cache, batch, out=planes), want)
            assert torch.equal(P.kv_attention(q[:, :1].expand(n, 4, 64), cache, batch), P.kv_attention(q[:, :1].expand(n, 4, 64).contiguous(), cache, batch))
            padded = torch.randn(n + 9, 4, 64, device="cuda").to(dtype)
            padded[4:n + 4] = q
            out, before = torch.full_like(padded, 7.0), padded.clone()
            P.kv_attention(padded, cache, P.KvBatch(batch.starts + 4, batch.lengths, batch.pages), out=out)
            assert torch.equal(out[4:n + 4], want) and (out[:4] == 7).all() and (out[n + 4:] == 7).all() and torch.equal(padded, before)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_masks_that_leave_a_row_empty(P, dtype):
    """No prefix and no bits; bits of tokens that are not there; a sequence shorter than its new tokens; nothing but scores of -inf."""
    for new, lengths in (((3, 2), (3, 70)), ((40, 2), (40, 2)), ((90,), (90,))):
        case = Case(new, lengths, 1, 2, 64, 16, dtype)
        words = 2 if max(new) <= 64 else 3
        tree = torch.randint(-2 ** 63, 2 ** 63 - 1, (case.tokens, words), generator=case.g)
        tree[0] = 0
        tree[-1] = -1
        tree[1] = 1 << 1
        check(run(P, case, tree), *attend(case, tree))
        assert (run(P, case, torch.zeros_like(tree))[:new[0]] == 0).all() or lengths[0] > new[0]
    case = Case((5, 1), (40, 9), 2, 1, 64, 16, dtype)
    cache, batch, q = case.device(P)
    batch.lengths.copy_(torch.tensor([2, 0], dtype=torch.int32))        # three of five tokens have no row, and see nothing
    got = P.kv_attention(q, cache, batch)
    assert (got[:3] == 0).all() and (got[5] == 0).all() and torch.isfinite(got).all()
    case.lengths, case.new, case.starts = [2], [2], torch.tensor([3, 5])
    want, lim = attend(case)
    check(got[3:5], want[3:5], lim[3:5])
    case = Case((1, 3), (40, 3), 1, 1, 64, 16, dtype)
    case.keys[torch.isfinite(case.keys)] = -torch.inf
    case.q.abs_()
    assert (run(P, case) == 0).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("new, length, at", [(4, 40, 37), (4, 4, 3), (70, 100, 60), (70, 70, 69), (200, 330, 300), (9, 1500, 1495)])
def test_what_is_not_seen_has_no_influence(P, dtype, bad, new, length, at):
    """A new token whose key and value are not finite: queries in front of it, or beside it in a tree, give what they gave; those that see it
    give what the definition gives."""
    case = Case((new,), (length,), 2, 2, 64, 16, dtype, seed=length)
    tree = trees(case, P)
    clean = run(P, case), run(P, case, tree)
    for where in ("values", "keys"):
        again = Case((new,), (length,), 2, 2, 64, 16, dtype, seed=length)
        rows = getattr(again, where)
        rows[again.table[0][at // 16], 0, at % 16, 3] = bad
        for mask, before in ((None, clean[0]), (tree, clean[1])):
            got = run(P, again, mask)
            from plain_kv import seen_of
            sees = seen_of(again, 0, mask)[:, at].cuda()
            assert torch.equal(got[~sees], before[~sees]) and torch.equal(got[:, 2:], before[:, 2:])
            if where == "values":
                expect = before[sees].clone()
                expect[:, :2, 3] = bad
                assert torch.equal(torch.nan_to_num(got[sees], 1e4, 2e4, 3e4), torch.nan_to_num(expect, 1e4, 2e4, 3e4))
            elif bad != bad:
                assert got[sees][:, :2].isnan().all()


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_pages_that_are_not_there(P, dtype):
    """Queries that see a row of a page out of range get NaN, the others what they got; nothing is read there."""
    for new, lengths in (((1, 1), (50, 130)), ((40, 3), (77, 130)), ((130, 1), (200, 20))):
        for number in (-1, 10 ** 9, -2 ** 31):
            case = Case(new, lengths, 1, 2, 64, 16, dtype)
            want = run(P, case)
            cache, batch, q = case.device(P)
            batch.pages[0, lengths[0] // 16 - 1] = number
            got = P.kv_attention(q, cache, batch)
            first = lengths[0] // 16 * 16 - 16
            sees = torch.arange(case.tokens, device="cuda") + lengths[0] - new[0] >= first
            sees[new[0]:] = False
            assert got[sees].isnan().all() and torch.equal(got[~sees], want[~sees])


def test_batches_whose_numbers_make_no_sense(P):
    """Whatever starts, lengths and pages hold, calls end and rows outside of sequences stay."""
    case = Case((3, 40, 1), (60, 50, 200), 2, 2, 64, 16, torch.bfloat16)
    cache, batch, q = case.device(P)
    for starts in ([0, 3, 2, 50], [-5, 10, 43, 44], [40, 30, 20, 10], [0, 2 ** 31 - 1, -2 ** 31, 7], [44, 44, 44, 44], [100, 200, 300, 400]):
        for lengths in ([60, 50, 200], [-1, -2 ** 31, 2 ** 31 - 1], [0, 0, 0], [2 ** 31 - 1] * 3):
            for pages in (batch.pages, torch.full_like(batch.pages, -7)):
                b = P.KvBatch(torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.tensor(lengths, dtype=torch.int32, device="cuda"), pages)
                P.kv_attention(q, cache, b)
                P.kv_append(cache, b, q[:, :2], q[:, 2:], q=q)
                P.kv_keep(cache, b, torch.tensor([[1, 2, 3], [0, 5, 4], [-1, 7, 2 ** 31 - 1]], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    empty = P.KvBatch(torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"),
                      torch.zeros(0, 4, dtype=torch.int32, device="cuda"))
    out = torch.ones_like(q)
    assert P.kv_attention(q, cache, empty, out=out) is not None and (out == 1).all()
    none = P.KvBatch(torch.zeros(4, dtype=torch.int32, device="cuda"), batch.lengths, batch.pages)
    assert P.kv_attention(q[:0], cache, none).shape == (0, 4, 64)
    assert (P.kv_attention(q, cache, P.KvBatch(batch.starts, batch.lengths, batch.pages[:, :0])) == 0).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_scales_and_large_scores(P, dtype):
    """Scores of hundreds, growing along the sequence (the running maximum moves at every tile) and shrinking; scales of zero and below."""
    case = Case((1, 50), (700, 300), 1, 2, 64, 16, dtype, spread=8.0)
    for scale in (None, 0.0, -0.3, 2.0):
        want, lim = attend(case, scale=scale)
        check(run(P, case, **({} if scale is None else dict(scale=scale))), want, lim)
    for sign in (1, -1):
        case = Case((1, 50), (700, 300), 1, 2, 64, 16, dtype, seed=5)
        case.q.fill_(0.5)
        for b, n in enumerate(case.lengths):
            for j in range(n):
                case.keys[case.table[b][j // 16], :, j % 16] = sign * j * 0.05
        check(run(P, case), *attend(case))


def test_far_rows_in_a_cache_past_32_bits(P):
    """A cache of more than 2^32 bytes, whose last pages are in use."""
    pages = 9000                                                        # 9000 x 8 x 128 x 256 x 2 bytes: 4.7e9 each
    keys = torch.empty(pages, 8, 128, 256, dtype=torch.bfloat16, device="cuda")
    values = torch.empty_like(keys)
    cache = P.KvCache(keys, values)
    small = Case((3, 1), (300, 130), 8, 1, 256, 128, torch.bfloat16)
    order = [8999, 0, 8500, 4321, 8998]
    at = iter(order)
    for b in range(2):
        for i, p in enumerate(small.table[b]):
            to = next(at)
            keys[to], values[to] = small.keys[p].cuda(), small.values[p].cuda()
            small.pages[b, i] = to
    batch = P.KvBatch(small.starts.cuda(), torch.tensor(small.lengths, dtype=torch.int32).cuda(), small.pages.cuda())
    check(P.kv_attention(small.q.cuda(), cache, batch), *attend(small))
    new = torch.randn(4, 8, 256, device="cuda").to(torch.bfloat16)
    P.kv_append(cache, batch, new, new)
    assert torch.equal(keys[8500, :, 41:44].transpose(0, 1), new[:3]) and torch.equal(values[8998, :, 1], new[3])
    assert P.kv_keep(cache, batch, torch.tensor([[0, 2], [-1, -1]], dtype=torch.int32, device="cuda")).tolist() == [299, 129]
    assert torch.equal(keys[8500, :, 42], new[2])


def test_other_streams_and_graphs(P):
    """On a stream of its own; captured, then replayed over other inputs, lengths and trees, with eager calls between."""
    case = Case((1, 30, 4), (300, 90, 2000), 2, 2, 64, 16, torch.bfloat16)
    cache, batch, q = case.device(P)
    tree = trees(case, P).cuda()
    new = torch.randn(35, 2, 64, device="cuda").to(torch.bfloat16)
    paths = torch.tensor([[0, -1, -1], [0, 3, 7], [1, 2, 3]], dtype=torch.int32, device="cuda")

    def step():
        turned = P.kv_append(cache, batch, new, new, table=table, q=q)
        return turned, P.kv_attention(turned, cache, batch), P.kv_attention(turned, cache, batch, tree=tree), P.kv_keep(cache, batch, paths)

    table = P.rotary_table(32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):                                                  # two graphs of one memory pool
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=graphs[0][0].pool() if graphs else None):
            got = step()
        graphs.append((graph, got))
    for k in range(4):
        q.normal_()
        new.normal_()
        tree[5, 0] = 1 << k
        batch.lengths.copy_(torch.tensor([250 + k, 40 + k, 1900 + 17 * k], dtype=torch.int32))
        for graph, got in graphs:
            graph.replay()
            torch.cuda.synchronize()
            mine = [t.clone() for t in got]
            for a, b in zip(mine, step()):
                assert torch.equal(a, b)
            torch.cuda.synchronize()


def test_random_shapes(P):
    rng = np.random.default_rng(11)
    for k in range(40):
        dtype = DTYPES[k % 3]
        batch = int(rng.integers(1, 6))
        new = [int(rng.choice([0, 1, 1, 2, 5, 17, 33, 64, 100])) for _ in range(batch)]
        lengths = [n + int(rng.choice([0, 0, 1, 15, 64, 333, 1100])) for n in new]
        if not sum(new):
            new[0], lengths[0] = 1, lengths[0] + 1
        case = Case(new, lengths, int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 8, 11])), 8 * int(rng.integers(1, 33)), int(rng.choice([1, 5, 16, 32, 50, 64])), dtype,
                    seed=k, order=list(ORDERS)[k % 3])
        tree = trees(case, P) if k % 2 else None
        check(run(P, case, tree), *attend(case, tree))
