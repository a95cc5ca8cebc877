"""Every form of the product in 4 microscaled bits (tests/mx4_rules.py) with sums of six slabs and more, results in place of the
residual and blocks that are not finite."""
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(__file__))
import mx4_rules                                    # noqa: E402

pytestmark = pytest.mark.gpu

GRID = [0, 0.5, 1, 1.5, 2, 3, 4, 6]

# form, m, n, k; of the two largest forms one tile a workgroup and several, with 6, 7, 9, 10 and 16 slabs of 256
SIZES = [(-1, 16, 3999, 2360), (-1, 3, 4001, 4096), (0, 49, 37, 2304), (0, 33, 2003, 1535), (1, 33, 8681, 1535), (1, 41, 7999, 2520), (2, 65, 8308, 1535),
         (2, 65, 8395, 4096), (3, 257, 7834, 1535), (3, 1031, 7338, 1752), (3, 1027, 7242, 2304), (3, 1028, 7359, 2520), (3, 908, 8292, 4096),
         (4, 1410, 8141, 1535), (4, 2690, 8614, 1752), (4, 2953, 7557, 2304), (4, 4240, 5253, 2520), (4, 3477, 6018, 4096)]


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
