"""Every form of the product in 4 microscaled bits (tests/mx4_rules.py) with sums of six slabs and more, results in place of the
residual, blocks that are not finite and scales of all sizes; and the sums of the two matrix instructions the forms use."""
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(__file__))
import mx4_rules                                    # noqa: E402

pytestmark = pytest.mark.gpu

GRID = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
HALF_STEP = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}       # relative to the value
TINY = {"float32": 2.0 ** -150, "bfloat16": 2.0 ** -134, "float16": 2.0 ** -25}         # half of the type's smallest step

# form, m, n, k; of the two largest forms one tile a workgroup and several, with 6, 7, 9, 10 and 16 slabs of 256
SIZES = [(-1, 16, 3999, 2360), (-1, 3, 4001, 4096), (0, 49, 37, 2304), (0, 33, 2003, 1535), (1, 33, 8681, 1535), (1, 41, 7999, 2520), (2, 65, 8308, 1535),
         (2, 65, 8395, 4096), (3, 257, 7834, 1535), (3, 1031, 7338, 1752), (3, 1027, 7242, 2304), (3, 1028, 7359, 2520), (3, 908, 8292, 4096),
         (4, 1410, 8141, 1535), (4, 2690, 8614, 1752), (4, 2953, 7557, 2304), (4, 4240, 5253, 2520), (4, 3477, 6018, 4096)]
# one of each for what does not depend on the number of tiles
ONE_OF_EACH = [SIZES[i] for i in (0, 3, 5, 6, 10, 15)]


@pytest.fixture(scope="module")
def P():
    import paper_2510_23264_amd as p
    return p


class Rows:
    """Codes and scale bytes [rows][k] on the device, as the library takes them and in 64 bits."""

    def __init__(self, P, g, rows, k, low, high, positive=False):
        import torch
        kp = -(-k // 256) * 256
        self.P, self.k = P, k
        self.code = torch.randint(0, 8, (rows, kp), generator=g, device="cuda", dtype=torch.uint8)
        if not positive:
            self.code |= torch.randint(0, 2, (rows, kp), generator=g, device="cuda", dtype=torch.uint8) << 3
        self.code[:, k:] = 0
        self.scale = torch.randint(low, high + 1, (rows, kp // 32), generator=g, device="cuda", dtype=torch.uint8)

    def held(self):
        return self.P.Mx4(self.code[:, 0::2] | self.code[:, 1::2] << 4, self.scale.clone(), self.k)

    def values(self):
        import torch
        grid = torch.tensor(GRID + [-v for v in GRID], dtype=torch.float64, device="cuda")
        scale = torch.exp2(self.scale.double() - 127)
        scale[self.scale == 255] = float("nan")
        return grid[self.code.long()] * scale.repeat_interleave(32, 1)


def generator(*seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(sum(v * 1009 ** i for i, v in enumerate(seed)) % (1 << 40))


@pytest.mark.parametrize("form, m, n, k", SIZES)
def test_long_sums_and_results_in_place_of_the_residual(P, form, m, n, k):
    """Scales of 1 and 1/2: products are multiples of 2^-4 of at most 36, bias and residual of 1/4 up to 16, so every partial sum of
    4096 of them (below 2^24 multiples) is a binary32 number and results are exact sums, rounded once.  The residual is elsewhere, the
    result itself, or other columns of its rows; what lies beside the result stays as it was."""
    import torch
    assert mx4_rules.form(m, n, k) == form
    g = generator(m, n, k)
    a, w = Rows(P, g, m, k, 126, 127), Rows(P, g, n, k, 126, 127)
    qa, qw = a.held(), w.held()
    sums = a.values() @ w.values().t()
    bias = torch.randint(-64, 64, (n,), generator=g, device="cuda").float() / 4
    assert torch.equal(P.mx4_gemm(qa, qw), sums.float())
    for t in (torch.float32, torch.bfloat16, torch.float16):
        res = torch.randint(-64, 64, (m, n), generator=g, device="cuda").to(t) / 4
        want = (sums + bias + res.double()).to(t)
        assert torch.equal(P.mx4_gemm(qa, qw, bias=bias, residual=res, dtype=t), want)
        here = res.clone()
        P.mx4_gemm(qa, qw, bias=bias, residual=here, out=here)
        assert torch.equal(here, want), t
        buf = torch.full((m + 2, n + 5), 9.0, dtype=t, device="cuda")
        out = buf[1:m + 1, 3:n + 3]
        out.copy_(res)
        P.mx4_gemm(qa, qw, bias=bias, residual=out, out=out)
        assert torch.equal(out, want), t
        out.fill_(9.0)
        assert (buf == 9.0).all()
        del buf, here, out
        both = torch.full((m, 2 * n + 1), 9.0, dtype=t, device="cuda")
        both[:, :n] = res
        P.mx4_gemm(qa, qw, bias=bias, residual=both[:, :n], out=both[:, n + 1:])
        assert torch.equal(both[:, n + 1:], want) and torch.equal(both[:, :n], res) and (both[:, n] == 9.0).all()


@pytest.mark.parametrize("form, m, n, k", SIZES)
def test_what_is_not_finite_stays_where_it_is(P, form, m, n, k):
    """Blocks that read as NaN in the first, a middle and the last row of either operand, infinities and NaN in the residual: exactly
    their rows, columns and elements of the result, and the exact sums everywhere else."""
    import torch
    assert mx4_rules.form(m, n, k) == form
    g = generator(m, n, k, 1)
    a, w = Rows(P, g, m, k, 126, 127), Rows(P, g, n, k, 126, 127)
    blocks = -(-k // 32)
    for rows, operand in ((m, a), (n, w)):
        for i, (row, block) in enumerate(((0, 0), (rows // 2, blocks // 2), (rows - 1, blocks - 1))):
            if rows > 3 or i == 1:
                operand.scale[row, block] = 255
                operand.code[row, block * 32:block * 32 + 32] = 0
    want = a.values() @ w.values().t()
    assert want.isnan().any() and want.isfinite().double().mean() > 0.6
    res = torch.zeros(m, n, device="cuda")
    res[m // 3, n // 3], res[m // 4, n - 2], res[m // 5, 1] = float("inf"), float("-inf"), float("nan")
    for t in (torch.float32, torch.bfloat16):
        for residual in (None, res.to(t)):
            expected = (want if residual is None else want + residual.double()).to(t)
            got = P.mx4_gemm(a.held(), w.held(), residual=residual, dtype=t)
            assert torch.equal(got.isnan(), expected.isnan())
            assert torch.equal(got.nan_to_num(0.0, float("inf"), float("-inf")), expected.nan_to_num(0.0, float("inf"), float("-inf")))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("form, m, n, k", SIZES)
def test_scales_of_all_sizes(P, form, m, n, k, dtype):
    """A block of 32 products under one pair of scales sums exactly (multiples of 1/4 of the scales' product, at most 1152 of
    it).  A binary32 addition of each block, of up to eight partial sums, of bias and residual is off by 2^-24 of what has been summed
    at most: K / 32 + 10 of them, in any order; one rounding to the result's type on top.  That is 2^-17 of the sum of magnitudes at
    K = 4096, where an adder that dropped the low digits of single products would lose up to 4096 times 2^-24."""
    import torch
    assert mx4_rules.form(m, n, k) == form
    t = getattr(torch, dtype)
    g = generator(m, n, k, 2)
    a, w = Rows(P, g, m, k, 112, 130), Rows(P, g, n, k, 100, 124)
    bias = torch.randn(n, generator=g, device="cuda")
    res = torch.randn(m, n, generator=g, device="cuda").to(t)
    av, wv = a.values(), w.values()
    want = av @ wv.t() + bias.double() + res.double()
    size = av.abs() @ wv.abs().t() + bias.double().abs() + res.double().abs()
    got = P.mx4_gemm(a.held(), w.held(), bias=bias, residual=res, dtype=t).double()
    adds = -(-k // 32) + 10
    bound = 1.001 * adds * 2.0 ** -24 * size                  # 1.001: the partial sums' own errors, less than adds * 2^-24 of them
    bound = bound + HALF_STEP[dtype] * (want.abs() + bound) + TINY[dtype]
    assert ((got - want).abs() <= bound).all(), ((got - want).abs() / bound).max()


@pytest.mark.parametrize("form, m, n, k", ONE_OF_EACH)
def test_sums_of_positive_products_are_not_biased(P, form, m, n, k):
    """All operands positive, scales 2^24 apart: an adder that drops digits is low by half a unit of 2^-24 of the sum or more for each
    block that needs rounding; one that rounds to nearest is right on average.  Each of at most K / 32 + 8 roundings is off by up to one
    unit to either side, so a result deviates by sqrt((K / 32 + 8) / 3) <= 5.4 units (K / 32 up to 79) and the mean of the 64 000 results of the
    smallest case by 0.02: a quarter is far outside."""
    import torch
    assert mx4_rules.form(m, n, k) == form
    g = generator(m, n, k, 3)
    a, w = Rows(P, g, m, k, 115, 127, True), Rows(P, g, n, k, 115, 127, True)
    want = a.values() @ w.values().t()
    assert m * n >= 60000 and -(-k // 32) <= 79
    error = (P.mx4_gemm(a.held(), w.held()).double() - want) / want * 2.0 ** 24
    assert (error != 0).double().mean() > 0.2                 # there was something to round
    assert abs(error.mean()) <= 0.25 and error.abs().max() <= 1.001 * (-(-k // 32) + 8)


@pytest.mark.parametrize("form, m, n", [(-1, 16, 2000), (0, 64, 2000)])          # the instruction of 128 and that of 64 elements
@pytest.mark.parametrize("at", [0, 255])
def test_one_dominant_product_among_small_ones(P, form, m, n, at):
    """36 against 224 positive products 2^d smaller.  Up to d = 16 everything is a multiple of 2^-18 and less than 2^24 of them,
    binary32 numbers throughout: nothing may be lost.  Beyond, every block of 32 may cost one rounding."""
    import torch
    assert mx4_rules.form(m, n, 256) == form
    for d in range(0, 34, 2):
        g = generator(m, at, d)
        pair = []
        for rows, down in ((m, d // 2), (n, d - d // 2)):
            r = Rows(P, g, rows, 256, 127 - down, 127 - down, True)
            r.code[:, at // 32 * 32:at // 32 * 32 + 32] = 0
            r.code[:, at] = 7
            r.scale[:, at // 32] = 127
            pair.append(r)
        want = pair[0].values() @ pair[1].values().t()
        got = P.mx4_gemm(pair[0].held(), pair[1].held()).double()
        if d <= 16:
            assert torch.equal(got, want), d
        assert ((got - want).abs() <= 1.001 * 8 * 2.0 ** -24 * want).all(), d


@pytest.mark.parametrize("form, m, n, k", ONE_OF_EACH)
def test_small_sums_onto_a_large_one(P, form, m, n, k):
    """The first slab of 256 elements 2^d larger than all others.  Multiples of 2^-d / 4, less than 2^24 of them up to d = 8 (256 products
    of 36 at most, and 1/256 of the others): exact.  Beyond, a rounding for each block."""
    import torch
    assert mx4_rules.form(m, n, k) == form
    for d in (0, 8, 12, 17, 20, 22, 24):
        g = generator(m, n, k, d)
        pair = []
        for rows, down in ((m, d // 2), (n, d - d // 2)):
            r = Rows(P, g, rows, k, 127 - down, 127 - down, True)
            r.scale[:, :8] = 127
            pair.append(r)
        want = pair[0].values() @ pair[1].values().t()
        got = P.mx4_gemm(pair[0].held(), pair[1].held()).double()
        if d <= 8:
            assert torch.equal(got, want), d
        assert ((got - want).abs() <= 1.001 * (-(-k // 32) + 8) * 2.0 ** -24 * want).all(), d


@pytest.mark.parametrize("form, m, n, k", ONE_OF_EACH)
def test_the_ends_of_the_range(P, form, m, n, k):
    """Scales whose product is 2^-145: products are multiples of 2^-147, subnormal or small, and sums of them below 2^24 such multiples
    exact.  One operand's scales at the top of the range and the other's at the bottom: exact as in the middle.  Positive sums
    beyond the range are infinite."""
    import torch
    assert mx4_rules.form(m, n, k) == form
    g = generator(m, n, k, 4)
    for low, high in ((127 - 73, 127 - 72), (254, 0), (1, 253)):
        a, w = Rows(P, g, m, k, low, low), Rows(P, g, n, k, high, high)
        assert torch.equal(P.mx4_gemm(a.held(), w.held()), (a.values() @ w.values().t()).float())
    a, w = Rows(P, g, m, k, 254, 254, True), Rows(P, g, n, k, 254, 254, True)
    got = P.mx4_gemm(a.held(), w.held())
    want = (a.values() @ w.values().t()).float()
    assert torch.equal(got, want) and want.isinf().all()
