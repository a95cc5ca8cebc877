"""Attention over a paged cache where its numbers could betray how a call was shared out: weights that round, values and scales at the ends of
their range.  Each on tiles of 16, 32 and 128 rows, whole and cut."""
import pytest
import torch

from plain_kv import Case

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
# a token, whole and cut; 17 to 32 rows a head, whole and cut; a tile of 128 rows and more, whole and cut
SHAPES = [((1,), (200,)), ((1,), (1500,)), ((20, 9), (60, 150)), ((20,), (1500,)), ((150,), (260,)), ((100,), (1500,))]


@pytest.fixture(scope="module")
def P():
    import paper_2510_23264_amd as p
    return p


def run(P, case, tree=None, **how):
    cache, batch, q = case.device(P)
    return P.kv_attention(q, cache, batch, tree=None if tree is None else tree.cuda(), **how)


def wide(case):
    """Lists of pages that have room for much more, with which calls may be cut."""
    case.pages = torch.nn.functional.pad(case.pages, (0, 4000), value=-1)
    return case


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("new, lengths", SHAPES)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_equal_values_are_the_answer(P, dtype, new, lengths, d):
    """Values that are one number c in a column: sum w c / sum w is c whatever 16-bit weights w are, if the same ones are summed.  Products w c
    are exact in fp32, sums of n terms of one sign off by n 2^-24 each: together 2^-12.4 for 1500 rows, and the next number of fp16 is 2^-11 away at
    least, so the nearest is c."""
    case = wide(Case(new, lengths, 2, 1, d, 16, dtype, seed=d))
    c = torch.randn(2, d, generator=case.g).to(dtype)
    case.values.copy_(torch.where(case.values.isnan(), case.values, c[None, :, None]))
    assert torch.equal(run(P, case).cpu(), c.expand(case.tokens, 2, d))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("group", [1, 20, 40])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_weights_are_divided_by_their_own_sum(P, dtype, group, d):
    """Two rows, scores t and 0: the answer is (w v_0 + v_1) / (w + 1) with w = exp(t) rounded to 16 bits, in both places.  Columns are left out whose
    sum cancels by more than 2^-4, and those that lie nearer than 2^-14 of themselves to the middle between two numbers of the dtype: two products,
    a sum, a quotient and the exponential are off by 2^-22 of their terms at most, 2^-18 of what is left."""
    t = -torch.linspace(0.03, 4.0, 60, dtype=torch.float64).to(dtype)
    p, half = t.double().exp(), torch.finfo(dtype).eps / 2
    w = p.to(dtype).double()
    step = torch.exp2(torch.floor(torch.log2(p))) * half * 2
    t, w = (x[((p - w).abs() / step < 0.45) & ((p - w).abs() / step > 0.2)] for x in (t, w))     # rounded by much, and surely
    n = len(t)
    assert n > 10
    case = Case([1] * n, [2] * n, 1, group, d, 16, dtype, seed=group)
    case.q.zero_()
    case.q[:, :, 0] = 1
    for b in range(n):
        rows = case.keys[case.table[b][0], 0, :2]
        rows.zero_()
        rows[0, 0] = t[b]
    v = torch.stack([case.values[case.table[b][0], 0, :2] for b in range(n)]).double()
    sums = w[:, None] * v[:, 0] + v[:, 1]
    want = sums / (w[:, None] + 1)
    clear = sums.abs() * 16 > (w[:, None] * v[:, 0]).abs() + v[:, 1].abs()
    for side in (1 - 2.0 ** -14, 1 + 2.0 ** -14):
        clear &= (want * side).to(dtype) == want.to(dtype)
    assert clear.double().mean() > 0.7
    got = run(P, case, scale=1.0).cpu()
    off = (got != want.to(dtype)[:, None]) & clear[:, None]
    assert not off.any(), (int(off.sum()), int(clear.sum()) * group)
