"""The operators on a paged cache on batches of many sequences, of equal ones, side by side on two streams, and what they refuse on the device.
The bounds are those of plain_kv."""
import pytest
import torch

from paper_2510_23264_amd.binding import PahqError
from plain_kv import Case, attend, check

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def P():
    import paper_2510_23264_amd as p
    return p


def run(P, case, **how):
    cache, batch, q = case.device(P)
    return P.kv_attention(q, cache, batch, **how)


# more sequences than a wave has lanes, and than there are ranges; one of them far longer than the others, or all short; many that are empty
@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("lengths, new", [
    ([7] * 40 + [5000] + [9] * 60, [1] * 101), ([1, 0, 300, 0, 2] * 60 + [2600], [1, 0, 2, 0, 1] * 60 + [3]), ([3] * 1100 + [1500, 1], [1] * 1102),
    ([0] * 700 + [900], [0] * 700 + [50]), ([40, 2000] * 70, [40, 1] * 70)], ids=["101", "301", "1102", "last", "140"])
def test_many_sequences(P, dtype, lengths, new):
    case = Case(new, lengths, 1, 2, 64, 16, dtype, seed=len(lengths))
    got = run(P, case)
    check(got, *attend(case))
    assert torch.equal(got, run(P, case))


# equal sequences: as many tiles as run at a time, somewhat more (which are cut), and several times as many
@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("count", [64, 65, 75, 330])
def test_equal_sequences(P, dtype, count):
    case = Case([1] * count, [290] * count, 4, 1, 64, 32, dtype, seed=count)
    check(run(P, case), *attend(case))


# the lists of pages have room for much more than there is, which the host cannot tell from long sequences
@pytest.mark.parametrize("new, lengths", [((1,), (70,)), ((20, 1), (20, 300)), ((150,), (260,)), ((0, 1), (0, 1)), ((64,), (1700,))])
def test_wide_lists_of_pages(P, new, lengths):
    case = Case(new, lengths, 2, 4, 128, 16, torch.bfloat16, seed=3)
    case.pages = torch.nn.functional.pad(case.pages, (0, 20000), value=-1)
    check(run(P, case), *attend(case))


def test_the_largest_batch(P):
    """65535 sequences of one token each: the one row it sees is its answer."""
    n, i32 = 65535, lambda t: t.to(torch.int32).cuda()                  # noqa: E731
    cache = P.KvCache.empty(n + 2, 1, 1, 8)
    cache.keys.fill_(float("nan"))
    cache.values.fill_(float("nan"))
    pages = torch.randperm(n + 2, generator=torch.Generator().manual_seed(1))[:n]
    batch = P.KvBatch(i32(torch.arange(n + 1)), i32(torch.ones(n)), i32(pages)[:, None])
    k, v, q = (torch.randn(n, heads, 8, device="cuda").to(torch.bfloat16) for heads in (1, 1, 3))
    P.kv_append(cache, batch, k, v)
    assert torch.equal(cache.keys[pages.cuda(), 0, 0], k[:, 0]) and int(cache.keys.isnan().any(-1).sum()) == 2
    assert torch.equal(P.kv_attention(q, cache, batch), v.expand(n, 3, 8))
    assert P.kv_keep(cache, batch, i32(torch.zeros(n, 1))).eq(1).all()
    with pytest.raises(PahqError):
        P.kv_attention(torch.cat([q, q[:1]]), cache, P.KvBatch(i32(torch.arange(n + 2)), i32(torch.ones(n + 1)), i32(torch.zeros(n + 1, 1))))


def test_two_streams_at_once(P):
    """Calls that run at the same time have workspaces of their own."""
    cases = [Case((1, 1), (6000, 200), 2, 4, 64, 16, torch.bfloat16, seed=1), Case((1, 90), (4000, 800), 2, 4, 64, 16, torch.bfloat16, seed=2)]
    held = [c.device(P) for c in cases]
    want = [P.kv_attention(q, cache, batch) for cache, batch, q in held]
    for c, w in zip(cases, want):
        check(w, *attend(c))
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, (cache, batch, q) in enumerate(held):
            with torch.cuda.stream(streams[i]):
                got[i].append(P.kv_attention(q, cache, batch))
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for g, w in zip(got, want) for x in g)


def test_gradients_are_refused_and_writes_are_seen(P):
    case = Case((3, 1), (40, 20), 2, 2, 64, 16, torch.float32)
    cache, batch, q = case.device(P)
    k = torch.randn(4, 2, 64, device="cuda")
    leaf = q.clone().requires_grad_()
    for call in (lambda: P.kv_attention(leaf, cache, batch), lambda: P.kv_append(cache, batch, k.clone().requires_grad_(), k), lambda: P.kv_append(cache, batch, k, k, q=leaf),
                 lambda: P.kv_attention(q, P.KvCache(cache.keys, cache.values.clone().requires_grad_()), batch), lambda: P.kv_attention(q, cache, batch, out=leaf)):
        with pytest.raises(ValueError, match="gradient"):
            call()
    with torch.no_grad():
        assert torch.equal(P.kv_attention(leaf, cache, batch), P.kv_attention(q, cache, batch))
    import torch.autograd.forward_ad as fwd
    with fwd.dual_level(), pytest.raises(ValueError, match="tangent"):
        P.kv_attention(fwd.make_dual(q, q), cache, batch)
    # autograd's record of who wrote a tensor: what was saved for a backward pass does not pass for what it was
    out, before = torch.empty_like(q), cache.keys._version
    version = out._version
    P.kv_append(cache, batch, k, k)
    P.kv_attention(q, cache, batch, out=out)
    assert cache.keys._version > before and out._version > version
    before = cache.values._version
    P.kv_keep(cache, batch, torch.tensor([[0, 2], [-1, -1]], dtype=torch.int32, device="cuda"))
    assert cache.values._version > before
    with torch.inference_mode():
        assert P.kv_attention(q, cache, batch).isfinite().all()
