"""Forward-mode derivatives through the operators on device tensors: rotation carries a tangent, the others refuse one; none
is lost without a word."""
import numpy as np
import pytest


@pytest.fixture(scope="module")
def P():
    import paper_2510_23264_amd as p
    return p


def test_a_tangent_is_refused_before_anything_else():
    import torch
    import torch.autograd.forward_ad as forward
    import paper_2510_23264_amd as P
    with forward.dual_level():
        x = forward.make_dual(torch.zeros(4, 64), torch.ones(4, 64))
        with pytest.raises(ValueError, match="tangent"):
            P.mx4_quantize(x)
        with pytest.raises(ValueError, match="out: not where"):          # the primal alone would turn, under the tangent of before
            P.rotary(x.view(4, 1, 64), torch.zeros(4, dtype=torch.int64), P.rotary_table(32, device="cpu"), out=x.view(4, 1, 64))
        y = x.view(4, 1, 64)
        with torch.no_grad(), pytest.raises(ValueError, match="out: not where"):
            P.rotary(y, torch.zeros(4, dtype=torch.int64), P.rotary_table(32, device="cpu"), out=y)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotation_carries_a_tangent(P, layout, inverse):
    """The rotation is linear, so the tangent turns as the values do: the same kernel, the same bits.  And against a central
    difference in 64 bits of the fp32 results, whose two roundings (of sums of two products, magnitude 1.5) are what they differ by."""
    import torch
    import torch.autograd.forward_ad as forward
    torch.manual_seed(8)
    table, pos = P.rotary_table(24, 100.0), torch.tensor([0, 3, 1000, 70000, -9], device="cuda")
    how = dict(layout=layout, magnitude=1.5, inverse=inverse)
    x, v = torch.randn(5, 3, 32, device="cuda"), torch.randn(5, 3, 32, device="cuda")
    want, turned = P.rotary(x, pos, table, **how), P.rotary(v, pos, table, **how)
    for tangent in (v, v.transpose(1, 2).contiguous().transpose(1, 2)):
        for wrap in (torch.enable_grad, torch.no_grad):
            with wrap(), forward.dual_level():
                y, dy = forward.unpack_dual(P.rotary(forward.make_dual(x, tangent), pos, table, **how))
            assert torch.equal(y, want) and dy is not None and torch.equal(dy, turned)
    diff = (P.rotary(x + 4 * v, pos, table, **how).double() - P.rotary(x - 4 * v, pos, table, **how).double()) / 8
    size = 2 * 1.5 * (x.abs() + 4 * v.abs()).double().amax()
    assert ((diff - turned.double()).abs() <= 8 * 2.0 ** -23 * size).all()
    # a tangent of what a backward pass is given, and a gradient beside the tangent
    w = torch.randn(5, 3, 32, device="cuda", requires_grad=True)
    back = P.rotary(v, pos, table, layout=layout, magnitude=1.5, inverse=not inverse)
    with forward.dual_level():
        y = P.rotary(w, pos, table, **how)
        (g,) = torch.autograd.grad(y, w, forward.make_dual(x, v), create_graph=True)
        assert torch.equal(forward.unpack_dual(g).tangent, back)
        both = P.rotary(forward.make_dual(w, v), pos, table, **how)
        assert torch.equal(forward.unpack_dual(both).tangent, turned)
        assert torch.equal(torch.autograd.grad(forward.unpack_dual(both).primal, w, v)[0], back)


@pytest.mark.gpu
def test_the_others_refuse_a_tangent(P):
    import torch
    import torch.autograd.forward_ad as forward
    q = P.mx4_quantize(torch.randn(4, 64, device="cuda"))
    plain, bias = torch.randn(4, 4, device="cuda"), torch.zeros(4, device="cuda")
    table, pos = P.rotary_table(32), torch.arange(4, device="cuda")
    x = torch.randn(4, 3, 64, device="cuda")
    with forward.dual_level():
        dual = lambda t: forward.make_dual(t, torch.ones_like(t))      # noqa: E731
        for call in (lambda: P.mx4_quantize(dual(plain)), lambda: P.mx4_gemm(q, q, bias=dual(bias)), lambda: P.mx4_gemm(q, q, residual=dual(plain)),
                     lambda: P.mx4_gemm(q, q, out=dual(plain)), lambda: P.mx4_dequantize(q, out=dual(torch.zeros(4, 64, device="cuda"))),
                     lambda: P.rotary(dual(x), pos, table, out=x), lambda: P.rotary(x, pos, table, out=dual(x.clone()))):
            before = plain.clone(), x.clone()
            with pytest.raises(ValueError):
                call()
            assert torch.equal(plain, before[0]) and torch.equal(x, before[1])
        assert np.isfinite(P.mx4_gemm(q, q, bias=bias, residual=plain).cpu().numpy()).all()      # inside a level, without a tangent
        primal = forward.unpack_dual(dual(plain)).primal
        assert P.mx4_quantize(primal.detach()).rows == 4
