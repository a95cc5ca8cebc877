"""The operators on a paged cache as far as a machine without a GPU can see: what they refuse before anything is enqueued, and masks of
drafted trees."""
import ctypes as C

import pytest

EINVAL, ETOOBIG = -1, -7
A = 1 << 24                        # addresses that are only compared
HUGE = (1 << 31) - 1
CACHE = dict(keys=A, values=2 * A, dtype=1, pages=10, page_size=16, heads=2, d_head=64, page_stride=2048, head_stride=1024, slot_stride=64)
BATCH = dict(starts=3 * A, lengths=4 * A, pages=5 * A, batch=3, width=4, ld_pages=4, tokens=8)
ROWS = dict(k=(6 * A, 128, 64), v=(7 * A, 128, 64), q=(8 * A, 256, 64), out=(9 * A, 256, 64))


@pytest.fixture(scope="module")
def P():
    import paper_2510_23264_amd as p
    return p


def structs(P, change):
    from paper_2510_23264_amd.binding import KvBatchArg, KvCacheArg, KvRowsArg
    cache = KvCacheArg(**{n: change.pop("cache_" + n, v) for n, v in CACHE.items()})
    batch = KvBatchArg(**{n: change.pop("batch_" + n, v) for n, v in BATCH.items()})
    rows = {n: KvRowsArg(*r) if r else None for n, r in ((n, change.pop(n, v)) for n, v in ROWS.items())}
    return C.byref(cache), C.byref(batch), {n: C.byref(r) if r else None for n, r in rows.items()}


def append(P, **change):
    cache, batch, r = structs(P, change)
    a = dict(dict(positions=10 * A, table=11 * A, rot=32, layout=0, magnitude=1.0, q_heads=4), **change)
    return P.lib().pahq_kv_append(None, cache, batch, r["k"], r["v"], a["positions"], a["table"], a["rot"], a["layout"], a["magnitude"], r["q"], a["q_heads"], r["out"])


def attention(P, **change):
    change = dict(dict(batch_width=400, batch_ld_pages=400), **change)             # long enough to be cut, which takes a workspace
    cache, batch, r = structs(P, change)
    a = dict(dict(tree=None, words=0, scale=1.0, q_heads=4, workspace=12 * A, bytes=A), **change)
    return P.lib().pahq_kv_attention(None, cache, batch, r["q"], a["q_heads"], a["tree"], a["words"], a["scale"], r["out"], a["workspace"], a["bytes"])


def keep(P, **change):
    cache, batch, _ = structs(P, change)
    a = dict(dict(paths=13 * A, depth=5, after=14 * A), **change)
    return P.lib().pahq_kv_keep(None, cache, batch, a["paths"], a["depth"], a["after"])


CACHES = [(dict(cache_dtype=3), EINVAL), (dict(cache_pages=0), EINVAL), (dict(cache_page_size=0), EINVAL), (dict(cache_heads=0), EINVAL), (dict(cache_d_head=0), EINVAL),
          (dict(cache_d_head=60), EINVAL), (dict(cache_d_head=264, cache_slot_stride=264), EINVAL), (dict(cache_keys=None), EINVAL), (dict(cache_values=None), EINVAL),
          (dict(cache_keys=A + 8), EINVAL), (dict(cache_values=2 * A + 4), EINVAL), (dict(cache_page_stride=-2048), EINVAL), (dict(cache_head_stride=1028), EINVAL),
          (dict(cache_slot_stride=56), EINVAL), (dict(cache_slot_stride=32), EINVAL), (dict(cache_head_stride=1016), EINVAL), (dict(cache_page_stride=2040), EINVAL),
          (dict(cache_head_stride=0), EINVAL), (dict(cache_values=A), EINVAL), (dict(cache_values=A + 128), EINVAL), (dict(cache_values=A + 2048), EINVAL),
          (dict(cache_page_stride=1 << 60), EINVAL), (dict(cache_page_stride=1 << 62), EINVAL), (dict(cache_slot_stride=1 << 52), EINVAL), (dict(cache_heads=65536, cache_page_stride=1 << 30), ETOOBIG)]
BATCHES = [(dict(batch_batch=-1), EINVAL), (dict(batch_width=-1), EINVAL), (dict(batch_tokens=-1), EINVAL), (dict(batch_starts=None), EINVAL),
           (dict(batch_lengths=None), EINVAL), (dict(batch_pages=None), EINVAL), (dict(batch_starts=3 * A + 2), EINVAL), (dict(batch_lengths=4 * A + 1), EINVAL),
           (dict(batch_pages=5 * A + 3), EINVAL), (dict(batch_width=400, batch_ld_pages=399), EINVAL), (dict(batch_ld_pages=1 << 62), EINVAL), (dict(batch_batch=65536), ETOOBIG)]


@pytest.mark.parametrize("change, code", CACHES + BATCHES)
def test_a_cache_or_a_batch_that_does_not_fit(P, change, code):
    assert append(P, **change) == attention(P, **change) == keep(P, **change) == code
    n = C.c_size_t()
    left = dict(change)
    cache, batch, _ = structs(P, left)
    assert P.lib().pahq_kv_attention_workspace(cache, batch, 4, C.byref(n)) == code


@pytest.mark.parametrize("change, code", [
    (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(q=None), EINVAL), (dict(out=None), EINVAL), (dict(k=(None, 128, 64)), EINVAL), (dict(v=(7 * A + 1, 128, 64)), EINVAL),
    (dict(k=(6 * A, -128, 64)), EINVAL), (dict(k=(6 * A, 1 << 62, 64)), EINVAL), (dict(q_heads=0), EINVAL), (dict(rot=0), EINVAL), (dict(rot=33), EINVAL), (dict(rot=66), EINVAL), (dict(layout=2), EINVAL),
    (dict(positions=10 * A + 4), EINVAL), (dict(table=11 * A + 4), EINVAL), (dict(out=(9 * A, 255, 64)), EINVAL), (dict(out=(9 * A, 256, 63)), EINVAL), (dict(out=(9 * A, 0, 64)), EINVAL),
    (dict(out=(8 * A + 2, 256, 64)), EINVAL), (dict(out=(8 * A, 512, 64)), EINVAL), (dict(out=(6 * A, 256, 64)), EINVAL), (dict(out=(7 * A + 128, 256, 64)), EINVAL),
    (dict(out=(A, 256, 64)), EINVAL), (dict(k=(A + 64, 128, 64)), EINVAL), (dict(q=(2 * A, 256, 64)), EINVAL), (dict(out=(10 * A, 256, 64)), EINVAL),
    (dict(out=(11 * A, 256, 64)), EINVAL), (dict(out=(3 * A, 256, 64)), EINVAL), (dict(out=(4 * A, 256, 64)), EINVAL), (dict(out=(5 * A, 256, 64)), EINVAL), (dict(table=A), EINVAL),
    (dict(cache_keys=5 * A), EINVAL), (dict(q_heads=65536, q=(8 * A, 1 << 23, 64), out=(9 * A, 1 << 23, 64)), ETOOBIG), (dict(batch_tokens=1 << 24), ETOOBIG),
    (dict(batch_batch=0, k=None), 0), (dict(batch_tokens=0, v=None), 0)])
def test_append_refuses(P, change, code):
    if change.get("batch_batch") == 0 or change.get("batch_tokens") == 0:
        change = dict(change, batch_starts=None)
        if "batch_tokens" in change:
            change["batch_starts"] = 3 * A
    assert append(P, **change) == code


@pytest.mark.parametrize("change, code", [
    (dict(q=None), EINVAL), (dict(out=None), EINVAL), (dict(q_heads=0), EINVAL), (dict(q_heads=3), EINVAL), (dict(tree=15 * A, words=0), EINVAL), (dict(words=-1), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(scale=float("nan")), EINVAL),
    (dict(tree=15 * A + 4, words=1), EINVAL), (dict(q=(8 * A + 1, 256, 64)), EINVAL), (dict(q=(8 * A, -1, 64)), EINVAL), (dict(out=(9 * A, 255, 64)), EINVAL),
    (dict(out=(8 * A + 2, 256, 64)), EINVAL), (dict(out=(A, 256, 64)), EINVAL), (dict(out=(2 * A, 256, 64)), EINVAL), (dict(out=(3 * A, 256, 64)), EINVAL),
    (dict(out=(5 * A, 256, 64)), EINVAL), (dict(tree=9 * A, words=1), EINVAL), (dict(out=(12 * A, 256, 64)), EINVAL), (dict(workspace=A), EINVAL), (dict(workspace=8 * A), EINVAL),
    (dict(workspace=5 * A), EINVAL), (dict(workspace=None), EINVAL),
    (dict(bytes=4096), EINVAL), (dict(workspace=12 * A + 8), EINVAL), (dict(tree=12 * A, words=1), EINVAL), (dict(q_heads=131072, q=(8 * A, 1 << 24, 64), out=(9 * A, 1 << 24, 64)), ETOOBIG),
    (dict(batch_tokens=1 << 24), ETOOBIG), (dict(batch_tokens=0, q=None, out=None), 0)])
def test_attention_refuses(P, change, code):
    assert attention(P, **change) == code


@pytest.mark.parametrize("scale", [2.36e38, 3e38, -2.36e38, -3.4e38])
def test_attention_refuses_scales_that_overflow(P, scale):
    """Finite, but not what the scores are multiplied by: scale * log2 e, in fp32, is at most 3.4028e38."""
    assert attention(P, scale=scale) == EINVAL
    # what does not overflow gets as far as the next check, of the workspace
    assert attention(P, scale=2.358e38, workspace=None) == EINVAL and attention(P, scale=scale, batch_tokens=0) == EINVAL
    assert attention(P, scale=2.358e38, batch_tokens=0) == 0


@pytest.mark.parametrize("tokens, heads, group, batch", [(65535, 2, 32767, 1), (16448, 65280, 1, 16448), ((1 << 24) - 1, 129, 1, 1)])
def test_tiles_beyond_a_launch_are_too_big_for_the_workspace_too(P, tokens, heads, group, batch):
    """2^24 tiles and more: the size of the workspace is refused as the call is."""
    q_heads = heads * group
    rows = (8 * A, q_heads * 64, 64)
    change = dict(cache_heads=heads, cache_head_stride=1024, cache_page_stride=1024 * heads, cache_values=1 << 40, batch_batch=batch, batch_tokens=tokens, q_heads=q_heads,
                  q=rows, out=(1 << 52,) + rows[1:], batch_starts=1 << 41, batch_lengths=1 << 42, batch_pages=1 << 43, workspace=1 << 44)
    assert attention(P, **dict(change)) == ETOOBIG
    left = dict(change)
    cache, batch_arg, _ = structs(P, left)
    n = C.c_size_t()
    assert P.lib().pahq_kv_attention_workspace(cache, batch_arg, q_heads, C.byref(n)) == ETOOBIG


@pytest.mark.parametrize("change, code", [
    (dict(paths=None), EINVAL), (dict(after=None), EINVAL), (dict(depth=-1), EINVAL), (dict(paths=13 * A + 2), EINVAL), (dict(after=14 * A + 1), EINVAL), (dict(after=4 * A), EINVAL),
    (dict(after=3 * A + 8), EINVAL), (dict(after=5 * A), EINVAL), (dict(after=13 * A + 12), EINVAL), (dict(after=A), EINVAL), (dict(paths=2 * A), EINVAL), (dict(batch_batch=0, paths=None, after=None), 0)])
def test_keep_refuses(P, change, code):
    assert keep(P, **change) == code


def test_masks_of_trees(P):
    import torch
    assert P.tree_words([]).shape == (0, 1)
    assert P.tree_words([-1, 0, 0, 1, 2, -1, 3]).tolist() == [[1], [3], [5], [11], [21], [32], [75]]
    chain = P.tree_words(range(-1, 129))
    assert chain.shape == (130, 3) and chain[129].tolist() == [2 ** 64 - 1, 2 ** 64 - 1, 3] and chain[63].tolist() == [2 ** 64 - 1, 0, 0]
    bits = P.tree_bits(list(range(-1, 69)), device="cpu")
    assert bits.dtype == torch.int64 and bits[69].tolist() == [-1, 63]
    for bad in ([0], [-1, 1], [-2], [-1, 0, 3]):
        with pytest.raises(P.PahqError):
            P.tree_words(bad)
    with pytest.raises(ValueError):
        P.tree_words([[-1]])
    assert P.lib().pahq_tree_bits(None, 1, None) == EINVAL and P.lib().pahq_tree_bits(None, -1, None) == EINVAL


def test_parents_are_whole_numbers_that_are_nodes(P):
    """Numbers that 32 bits would turn into others, and fractions that would be cut off."""
    import numpy as np
    for bad in (np.array([2 ** 32 - 1]), np.array([-1, 2 ** 32]), np.array([-1, -2 ** 32 - 1]), np.array([2 ** 64 - 1], dtype=np.uint64)):
        with pytest.raises(P.PahqError):
            P.tree_words(bad)
    for bad in ([-1.0, 0.5], [-1, None], ["-1"], [True, False], -1):
        with pytest.raises(ValueError):
            P.tree_words(bad)
    assert P.tree_words(np.array([-1, 0], dtype=np.int64)).tolist() == P.tree_words(np.array([-1, 0], dtype=np.int8)).tolist() == [[1], [3]]


def test_the_quotient_of_a_page_size_is_exact():
    """j / p as a product and a shift: at the multiples' borders, for every size a shift's range turns on, and at random."""
    import random
    rng = random.Random(1)
    sizes = [1, 2, 3, 5, 7, 16, 24, 48, 100, 255, 256, 257, 65535, 65537, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, HUGE] + [rng.randrange(1, HUGE) for _ in range(300)]
    for p in sizes:
        s = (p - 1).bit_length()
        magic = ((1 << 31 + s) + p - 1) // p
        assert magic < 1 << 32
        for j in [0, 1, p - 1, p, HUGE, HUGE // p * p, HUGE // p * p - 1] + [rng.randrange(HUGE) for _ in range(50)] + [rng.randrange(HUGE // p + 1) * p for _ in range(50)]:
            if 0 <= j <= HUGE:
                assert j * magic >> 31 + s == j // p, (j, p)


def test_wrappers_refuse_host_tensors_and_shapes(P):
    import torch
    keys = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)                 # noqa: E731
    cache, batch, q = P.KvCache(keys, keys.clone()), P.KvBatch(i32(3), i32(2), i32(2, 4)), torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    for call in (lambda: P.kv_attention(q, cache, batch), lambda: P.kv_append(cache, batch, q[:, :2], q[:, 2:]), lambda: P.kv_keep(cache, batch, i32(2, 3)),
                 lambda: P.KvCache(keys, keys[:2]), lambda: P.KvCache(keys, keys.float()), lambda: P.KvCache(keys[0], keys[0]), lambda: P.KvCache(keys.int(), keys.int()),
                 lambda: P.KvBatch(i32(2), i32(2), i32(2, 4)), lambda: P.KvBatch(i32(3), i32(2), i32(3, 4)), lambda: P.KvBatch(i32(3).long(), i32(2).long(), i32(2, 4).long()),
                 lambda: P.KvBatch(i32(3), i32(2), i32(8)), lambda: P.kv_append(cache, batch, q, q, layout="other")):
        with pytest.raises(ValueError):
            call()
