"""Attention over a paged cache where its numbers could betray how a call was shared out: weights that round, values and scales at the ends of
their range.  Each on tiles of 16, 32 and 128 rows, whole and cut."""
import pytest
import torch

from plain_kv import Case, attend, check, seen_of

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


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new, lengths", SHAPES)
@pytest.mark.parametrize("weight", ["small", "gone", "overtaken"])
def test_infinite_values_count_whatever_their_weight(P, dtype, d, new, lengths, weight):
    """A value that is infinite in one column of a row that every query sees, or in a new token's row that some see.  Its weight is exp(-25), which 16
    bits may not hold, or exp(-120), which fp32 does not hold, or it was exp(0) until later rows' scores of 120 took over: positive
    in the definition.  The column is infinite for those that see the row (NaN for both signs), and nothing else changes by a bit."""
    def made():
        case = wide(Case(new, lengths, 2, 1, d, 16, dtype, seed=sum(lengths)))
        case.q *= 0.0625
        case.q[:, :, 0] = 1
        there = ~case.keys[:, :, :, 0].isnan()
        case.keys[:, :, :, 0][there] = 0.0
        return case

    def row(case, name, j):
        return getattr(case, name)[case.table[0][j // 16], 0, j % 16]
    for at in (5, lengths[0] - max(1, new[0] // 2)):
        def prepared():
            case = made()
            if weight == "overtaken":
                for j in range(at + 1, lengths[0]):
                    case.keys[case.table[0][j // 16], :, j % 16, 0] = 120.0
            else:
                row(case, "keys", at)[0] = row(case, "keys", at - 1)[0] = -25.0 if weight == "small" else -120.0
            return case
        tree = torch.full((made().tokens, -(-max(new) // 64)), -1)
        tree[: new[0] // 2, (at - lengths[0] + new[0]) // 64 if at >= lengths[0] - new[0] else 0] = 0
        for mask in (None, tree):
            clean = run(P, prepared(), mask, scale=1.0).cpu()
            sees = seen_of(made(), 0, mask)[:, at - 1:at + 1]
            for first, second in ((float("inf"), 0.5), (0.5, -float("inf")), (float("inf"), -float("inf"))):
                case = prepared()
                row(case, "values", at - 1)[3], row(case, "values", at)[3] = first, second
                got = run(P, case, mask, scale=1.0).cpu()
                want = clean.clone()
                for i in range(new[0]):
                    bad = [x for x, s in zip((first, second), sees[i].tolist()) if s and abs(x) > 1]
                    if bad:
                        want[i, 0, 3] = sum(bad)
                    elif sees[i].any():
                        want[i, 0, 3] = got[i, 0, 3]                     # 0.5 where a number stood, of a weight that counts in the "overtaken" row
                        assert got[i, 0, 3].isfinite()
                assert torch.equal(torch.nan_to_num(got, 1e4, 2e4, 3e4), torch.nan_to_num(want, 1e4, 2e4, 3e4)), (at, mask is None, first, second)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("new, lengths", SHAPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_scale_of_zero_hides_no_query(P, dtype, new, lengths, bad):
    """Scores are 0 times the product: NaN where a query is not finite, its own rows only; 0 for the others, which get the values' mean."""
    case = wide(Case(new, lengths, 2, 1, 64, 16, dtype, seed=7))
    clean = run(P, case, scale=0.0).cpu()
    check(clean, *attend(case, scale=0.0))
    case.q[case.tokens // 2, 1, 17] = bad
    got = run(P, case, scale=0.0).cpu()
    assert got[case.tokens // 2, 1].isnan().all()
    got[case.tokens // 2, 1] = clean[case.tokens // 2, 1]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("new, lengths", SHAPES)
@pytest.mark.parametrize("d", [64, 128, 192, 256])
def test_the_same_call_gives_the_same_bits(P, dtype, new, lengths, d):
    """Trees and causal calls, over and over, with memory of other values where the workspace and results come to lie; in place too; and with an
    infinite value, for which tiles are done twice."""
    case = wide(Case(new, lengths, 2, 3, d, 16, dtype, seed=d))
    tree = torch.randint(-2 ** 63, 2 ** 63 - 1, (case.tokens, -(-max(new) // 64)), generator=case.g).cuda()
    cache, batch, q = case.device(P)
    for infinite in (False, True):
        if infinite:
            cache.keys[case.table[0][0], :, 2, :] = cache.keys[case.table[0][0], :, 2, :] * 16
            cache.values[case.table[0][0], :, 2, 5] = float("inf")
        for mask in (None, tree):
            first = P.kv_attention(q, cache, batch, tree=mask)
            for k in range(6):
                torch.full((1 << 22,), float(k), device="cuda")
                assert torch.equal(P.kv_attention(q, cache, batch, tree=mask), first)
            mine = q.clone()
            P.kv_attention(mine, cache, batch, tree=mask, out=mine)
            assert torch.equal(mine, first)
            assert infinite == bool((~first.isfinite()).any()) or (mask is not None and lengths[0] == new[0])


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("group", [1, 20, 40])
@pytest.mark.parametrize("low", [15, 18, 20, 21, 22, 23, 24, 25])
def test_many_small_weights_count_as_one_large_does(P, dtype, group, low):
    """One row of score 0 and 16000 of 2^-low each, that together weigh 0.5 to 2^-11 of it; values 0 there, 1 here.  fp16 holds a weight down to 2^-31 of
    the largest (2^-24 times 2^-7), some as numbers that are not normal, and the two sums have to take the same ones: sums of 16000 terms of one sign in
    fp32, off by 16000 2^-24 = 2^-10 each, a weight rounded by half a step of its own or by 2^-32 of the largest, half a step of the result."""
    n, d = 16001, 64
    case = Case([1], [n], 1, group, d, 64, dtype)
    case.q.zero_()
    case.q[:, :, 0] = 1
    there = ~case.keys[:, :, :, 0].isnan()
    case.keys[:, :, :, 0][there] = 0.0
    case.values[~case.values.isnan()] = 1.0
    x = torch.tensor(low * 0.6931471805599453).to(dtype)
    for j in range(0, n, 64):
        case.keys[case.table[0][j // 64], 0, :min(64, n - j), 0] = -x
    case.keys[case.table[0][100], 0, 5, 0] = 0.0
    case.values[case.table[0][100], 0, 5] = 0.0
    w = float(torch.exp(-x.double()))
    want = 16000 * w / (1 + 16000 * w)
    got = run(P, case, scale=1.0).double().cpu()
    u = torch.finfo(dtype).eps / 2
    lim = want * (2 * 2.0 ** -10 + 2 * u + (2.0 ** -32 / w if dtype == torch.float16 else 0.0))
    assert (got - want).abs().max() <= lim, (float(got.min()), float(got.max()), want, lim)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("new, lengths", SHAPES)
def test_large_values_do_not_overflow(P, dtype, new, lengths):
    """Values times 2^104 give 2^104 times the answer, every rounding being the same: values below 2^3 and lengths below 2^11 leave all sums below 2^128.
    Growing scores, with which weights are as large as they get."""
    case = wide(Case(new, lengths, 2, 1, 64, 16, dtype, seed=1))
    case.q[:, :, 0] = 1
    for b, n in enumerate(lengths):
        for j in range(n):
            case.keys[case.table[b][j // 16], :, j % 16, 0] = 0.125 * j
    assert case.values[~case.values.isnan()].abs().max() < 8
    plain = run(P, case)
    case.values *= 2.0 ** 104
    assert torch.equal(run(P, case), plain * 2.0 ** 104) and plain.isfinite().all()
