"""Strides that no memory has: refused before a product of theirs that passes 64 bits is taken for a small one."""
import pytest

from test_tensor_operators import A, DEQUANTIZE, EINVAL, GEMM, QUANTIZE, ROTARY

FAR = [1 << 62, 1 << 61, (1 << 63) - 1, (1 << 62) + 300, (1 << 60) + 100, 1 << 54]


@pytest.fixture(scope="module")
def lib():
    import paper_2510_23264_amd as P
    return P.lib()


@pytest.mark.parametrize("stride", FAR)
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_strides_past_64_bits(lib, stride, dtype):
    for name, base, changes in (
            ("pahq_mx4_quantize", QUANTIZE, [dict(ld=stride), dict(ld=stride, by=1)]), ("pahq_mx4_dequantize", DEQUANTIZE, [dict(ld=stride)]),
            ("pahq_mx4_gemm", GEMM, [dict(ld=stride), dict(ld_res=stride), dict(ld=stride, ld_res=stride, residual=7 * A)]),
            ("pahq_rotary", ROTARY, [dict(x_token=stride), dict(x_head=stride), dict(out_token=stride), dict(out_head=stride),
                                     dict(out_head=stride, out_token=64), dict(x_token=stride, x_head=stride),
                                     dict(x_token=stride, x_head=64, out=A, out_token=stride)])):
        for change in changes:
            assert getattr(lib, name)(*dict(base, dtype=dtype, **change).values()) == EINVAL, (name, change)


def test_negative_strides(lib):
    for change in (dict(x_head=-1), dict(out_token=-192), dict(out_head=-64), dict(tokens=1, out_token=-1), dict(heads=1, out_head=-1, x_head=-1)):
        assert lib.pahq_rotary(*dict(ROTARY, **change).values()) == EINVAL, change
