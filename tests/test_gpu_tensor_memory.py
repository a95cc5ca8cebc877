"""A result for which there is no memory: torch's own error, and the next call works."""
import pytest

pytestmark = pytest.mark.gpu


def test_results_larger_than_the_device():
    import torch
    import paper_2510_23264_amd as P
    q = P.mx4_quantize(torch.randn(1 << 21, 8, device="cuda"))
    wide = P.mx4_quantize(torch.randn(3, 8, device="cuda"))
    x = torch.randn(1, 1, 64, device="cuda")
    for call in (lambda: P.mx4_gemm(q, q),                                             # 2^42 results in fp32
                 lambda: P.rotary(x.expand(1 << 20, 1 << 15, 64), torch.zeros(1 << 20, dtype=torch.int64, device="cuda"), P.rotary_table(64))):
        with pytest.raises(torch.OutOfMemoryError):
            call()
    assert torch.equal(P.mx4_gemm(wide, wide), P.mx4_gemm(wide, wide)) and P.rotary(x, torch.zeros(1, dtype=torch.int64, device="cuda"), P.rotary_table(64)).shape == x.shape
