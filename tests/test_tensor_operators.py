"""The operators on device tensors as far as a machine without a GPU can see: what they refuse before anything is enqueued,
sizes, and the rotary table against frequencies in exact arithmetic."""
import ctypes as C
from fractions import Fraction
import math

import pytest

EINVAL, ETOOBIG = -1, -7
A = 1 << 20                        # addresses that are only compared
HUGE = (1 << 31) - 1


@pytest.fixture(scope="module")
def P():
    import paper_2510_23264_amd as p
    return p


def test_sizes_of_a_held_matrix(P):
    for rows, cols, k in ((0, 1, 256), (1, 1, 256), (3, 256, 256), (5, 257, 512), (HUGE, 4096, 4096)):
        c, s = C.c_size_t(), C.c_size_t()
        assert P.lib().pahq_mx4_bytes(rows, cols, C.byref(c), C.byref(s)) == 0
        assert (c.value, s.value) == (rows * k // 2, rows * k // 32)
    assert P.lib().pahq_mx4_bytes(-1, 4, C.byref(c), C.byref(s)) == EINVAL
    assert P.lib().pahq_mx4_bytes(1, 0, C.byref(c), C.byref(s)) == EINVAL
    assert P.lib().pahq_mx4_bytes(1, 1, None, C.byref(s)) == EINVAL


QUANTIZE = dict(stream=None, x=A, dtype=0, rows=4, cols=300, ld=300, by=0, codes=2 * A, scales=3 * A)
DEQUANTIZE = dict(stream=None, codes=2 * A, scales=3 * A, rows=4, cols=300, out=A, dtype=0, ld=300)
GEMM = dict(stream=None, a=A, a_scales=2 * A, w=3 * A, w_scales=4 * A, m=4, n=8, k=300, bias=5 * A, residual=6 * A, ld_res=8, out=7 * A, dtype=0, ld=8)
ROTARY = dict(stream=None, x=A, dtype=0, tokens=4, heads=3, d=64, x_token=192, x_head=64, positions=4 * A, table=5 * A, rot=32, layout=0, magnitude=1.0,
              inverse=0, out=2 * A, out_token=192, out_head=64)


@pytest.mark.parametrize("change, code", [
    (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(dtype=3), EINVAL), (dict(dtype=-1), EINVAL), (dict(by=2), EINVAL), (dict(ld=299), EINVAL),
    (dict(by=1, ld=3), EINVAL), (dict(x=None), EINVAL), (dict(codes=None), EINVAL), (dict(scales=None), EINVAL), (dict(codes=2 * A + 8), EINVAL),
    (dict(scales=3 * A + 4), EINVAL), (dict(x=A + 2), EINVAL), (dict(x=A + 1, dtype=1), EINVAL), (dict(codes=A + 16), EINVAL), (dict(scales=A + 16), EINVAL),
    (dict(scales=2 * A + 16), EINVAL), (dict(rows=HUGE, cols=513, ld=513), ETOOBIG), (dict(rows=1 << 27), ETOOBIG), (dict(by=1, cols=65535 * 256 + 1), ETOOBIG),
    (dict(rows=0, x=None), 0)])
def test_quantize_refuses(P, change, code):
    assert P.lib().pahq_mx4_quantize(*dict(QUANTIZE, **change).values()) == code


@pytest.mark.parametrize("change, code", [
    (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(dtype=7), EINVAL), (dict(ld=299), EINVAL), (dict(out=None), EINVAL), (dict(codes=None), EINVAL),
    (dict(codes=2 * A + 1), EINVAL), (dict(scales=3 * A + 1), EINVAL), (dict(out=A + 1), EINVAL), (dict(out=2 * A), EINVAL), (dict(out=3 * A), EINVAL),
    (dict(rows=HUGE), ETOOBIG), (dict(rows=0, out=None), 0)])
def test_dequantize_refuses(P, change, code):
    assert P.lib().pahq_mx4_dequantize(*dict(DEQUANTIZE, **change).values()) == code


@pytest.mark.parametrize("change, code", [
    (dict(m=-1), EINVAL), (dict(n=-1), EINVAL), (dict(k=0), EINVAL), (dict(dtype=3), EINVAL), (dict(ld=7), EINVAL), (dict(ld_res=7), EINVAL),
    (dict(a=None), EINVAL), (dict(a_scales=None), EINVAL), (dict(w=None), EINVAL), (dict(w_scales=None), EINVAL), (dict(out=None), EINVAL),
    (dict(a=A + 4), EINVAL), (dict(w_scales=4 * A + 2), EINVAL), (dict(out=7 * A + 2), EINVAL), (dict(residual=6 * A + 1), EINVAL), (dict(bias=5 * A + 2), EINVAL),
    (dict(out=A), EINVAL), (dict(out=2 * A), EINVAL), (dict(out=3 * A), EINVAL), (dict(out=4 * A), EINVAL), (dict(out=5 * A), EINVAL),
    (dict(residual=7 * A + 4), EINVAL), (dict(residual=7 * A, ld_res=9), EINVAL), (dict(n=HUGE, k=513, ld=HUGE, ld_res=HUGE), ETOOBIG), (dict(k=(1 << 24) + 1), ETOOBIG),
    (dict(n=1 << 27, k=64, ld=1 << 27, ld_res=1 << 27), ETOOBIG), (dict(residual=7 * A + 16, ld=14, ld_res=14), EINVAL), (dict(residual=7 * A + 64, ld=16, ld_res=17), EINVAL),
    (dict(m=0, a=None, out=None), 0), (dict(n=0, w=None, ld=0), 0)])
def test_gemm_refuses(P, change, code):
    assert P.lib().pahq_mx4_gemm(*dict(GEMM, **change).values()) == code


@pytest.mark.parametrize("change, code", [
    (dict(tokens=-1), EINVAL), (dict(heads=-1), EINVAL), (dict(d=0), EINVAL), (dict(dtype=4), EINVAL), (dict(rot=0), EINVAL), (dict(rot=31), EINVAL),
    (dict(rot=66), EINVAL), (dict(rot=1026, d=2048, x_head=2048, x_token=8192, out_head=2048, out_token=8192), EINVAL), (dict(layout=2), EINVAL),
    (dict(inverse=2), EINVAL), (dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(positions=None), EINVAL), (dict(table=None), EINVAL),
    (dict(x=A + 2), EINVAL), (dict(out=2 * A + 1), EINVAL), (dict(positions=4 * A + 4), EINVAL), (dict(table=5 * A + 4), EINVAL), (dict(x_token=-1), EINVAL),
    (dict(out_head=63), EINVAL), (dict(out_token=191), EINVAL), (dict(out_token=0), EINVAL), (dict(out_token=64, out_head=255), EINVAL),
    (dict(out=A + 4), EINVAL), (dict(out=A, out_token=256), EINVAL), (dict(out=4 * A), EINVAL), (dict(out=5 * A), EINVAL),
    (dict(heads=65536, out_token=1 << 28), ETOOBIG), (dict(tokens=1 << 24), ETOOBIG), (dict(d=4097, out_head=4097, out_token=3 * 4097), ETOOBIG), (dict(tokens=0, x=None), 0), (dict(heads=0, out=None), 0)])
def test_rotary_refuses(P, change, code):
    assert P.lib().pahq_rotary(*dict(ROTARY, **change).values()) == code


def table(P, rot, theta, scaling, factor=1.0, original=0.0, lo=1.0, hi=32.0):
    out = (C.c_uint64 * max(rot // 2, 1))()
    rc = P.lib().pahq_rotary_table(rot, theta, scaling, factor, original, lo, hi, out)
    return rc, list(out)


@pytest.mark.parametrize("rot, theta, scaling, factor", [(2, 10000.0, 0, 1.0), (64, 10000.0, 0, 1.0), (128, 500000.0, 1, 8.0), (96, 1e4, 2, 3.7),
                                                         (128, 1e6, 3, 8.0), (1024, 1e4, 3, 32.0), (4, 2.0, 2, 1.0)])
def test_table_holds_the_frequencies(P, rot, theta, scaling, factor):
    """Against the formulas in doubles: a double's frequency carries 2^-53 of itself a few times over, and an entry, a whole
    number of 2^-64, is off by half of one."""
    original, lo, hi = 8192.0, 1.0, 4.0
    rc, got = table(P, rot, theta, scaling, factor, original, lo, hi)
    assert rc == 0
    for i, t in enumerate(got):
        f = theta ** (-2.0 * i / rot)
        if scaling == 1:
            f /= factor
        if scaling == 2:
            f = (theta * factor ** (rot / (rot - 2))) ** (-2.0 * i / rot)
        if scaling == 3:
            r = original * f / (2 * math.pi)
            f = f / factor if r <= lo else f if r >= hi else f * ((r - lo) / (hi - lo) + (1 - (r - lo) / (hi - lo)) / factor)
        assert abs(float(Fraction(t, 1 << 64)) - f / (2 * math.pi)) <= 2.0 ** -65 + 2.0 ** -48 * f, i


def test_table_ends_and_refusals(P):
    _, plain = table(P, 64, 10000.0, 0)
    _, base = table(P, 64, 10000.0, 2, 8.0)
    assert base[0] == plain[0] and abs(base[-1] * 8 - plain[-1]) <= 2.0 ** -40 * plain[-1]      # slowest stretched by 8, fastest kept
    assert table(P, 64, 10000.0, 3, 8.0, 4096.0)[1][0] == plain[0]
    for bad in ((0, 1e4, 0), (3, 1e4, 0), (1026, 1e4, 0), (64, 0.0, 0), (64, -1.0, 0), (64, math.inf, 0), (64, math.nan, 0), (64, 1e4, 4), (64, 1e4, -1),
                (64, 1e4, 1, 0.5), (64, 1e4, 1, math.nan), (2, 1e4, 2, 2.0), (64, 1e4, 3, 2.0, 0.0), (64, 1e4, 3, 2.0, math.nan), (64, 1e4, 3, 2.0, 10.0, 4.0, 4.0),
                (64, 1e4, 3, 2.0, 10.0, -1.0, 4.0)):
        assert table(P, *bad)[0] == EINVAL, bad
    assert P.lib().pahq_rotary_table(64, 1e4, 0, 1.0, 0.0, 1.0, 2.0, None) == EINVAL


def test_wrapper_refuses_host_tensors(P):
    import torch
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        P.mx4_quantize(x)
    with pytest.raises(ValueError):
        P.Mx4(torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 8, dtype=torch.uint8), 64)
    with pytest.raises(ValueError):
        P.rotary(x.view(4, 1, 64), torch.zeros(4, dtype=torch.int64), P.rotary_table(32, device="cpu"))
    with pytest.raises(ValueError):
        P.rotary_table(32, scaling="other", device="cpu")
    with pytest.raises(P.PahqError):
        P.rotary_table(31, device="cpu")
