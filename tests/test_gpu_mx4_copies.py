"""Copies of a matrix in 4 microscaled bits do not see what is written into the one they come from."""
import copy

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [5, 1, 0])
def test_a_shallow_copy_has_memory_of_its_own(rows):
    import torch
    import paper_2510_23264_amd as P
    x, w = torch.randn(rows, 300, device="cuda"), P.mx4_quantize(torch.randn(7, 300, device="cuda"))
    made = P.mx4_quantize(x)
    given = P.Mx4(made.codes.clone(), made.scales.clone(), 300)
    for q in (made, given):
        want = P.mx4_gemm(q, w)
        c = copy.copy(q)
        assert (c.rows, c.cols, c.device) == (rows, 300, q.device)
        P.mx4_quantize(torch.zeros_like(x), out=q)
        assert not P.mx4_gemm(q, w).any()
        assert torch.equal(P.mx4_gemm(c, w), want)
        d = copy.deepcopy(c)
        P.mx4_quantize(torch.zeros_like(x), out=c)
        assert torch.equal(P.mx4_gemm(d, w), want)
