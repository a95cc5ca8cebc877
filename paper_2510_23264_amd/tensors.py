"""The library's operators on device tensors (include/pahq.h, the section of that name) with torch tensors: matrices
in 4 microscaled bits and their product, and rotary positions.

Every call enqueues on the current stream of its tensors' device (whichever device is current) and does not wait.  Results are
new tensors unless `out` is given.  Strided tensors are taken as they are where the C functions can walk them and refused
otherwise; nothing is copied behind the caller's back.  Arguments that do not fit raise ValueError, a refusal of the
library raises PahqError."""
from __future__ import annotations

import numpy as np
import torch

from .binding import lib, _chk, rotary_entries

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_LAYOUTS = {"half": 0, "interleaved": 1}


def _need(ok, what):
    if not ok:
        raise ValueError(what)


_functions = {}


def _call(name, device, *args):
    """One library call on the current stream of `device`, with that device current.  (The function kept and the stream asked for as
    a number: a small call takes the host 7 us instead of 9, of which the launch is 2.)"""
    fn = _functions.get(name)
    if fn is None:
        fn = _functions[name] = getattr(lib(), name)
    index = device.index
    if index == torch._C._cuda_getDevice():
        code = fn(torch._C._cuda_getCurrentRawStream(index), *args)
    else:
        with torch.cuda.device(device):
            code = fn(torch._C._cuda_getCurrentRawStream(index), *args)
    if code:
        _chk(code, name)


def _tracked(t):
    return t.requires_grad and torch.is_grad_enabled()


def _row_stride(t):
    """Elements from row to row of a matrix whose rows are contiguous; None if they are not.  Of a single row or column torch
    reports any stride."""
    rows, cols = t.shape
    if t.is_contiguous() or rows <= 1 and (cols <= 1 or t.stride(1) == 1):
        return cols or 1
    ld, step = t.stride()
    return ld if (step == 1 or cols <= 1) and ld >= cols else None


class Mx4:
    """A matrix [rows][cols] in 4 microscaled bits: `codes` uint8 [rows][K / 2] and `scales` uint8 [rows][K / 32], K = cols
    rounded up to 256, both contiguous on one device (the format is described in include/pahq.h)."""

    __slots__ = ("rows", "cols", "device", "_both", "_codes", "_scales", "_at")

    def __init__(self, codes, scales, cols):
        k = -(-int(cols) // 256) * 256
        _need(codes.dtype == scales.dtype == torch.uint8 and codes.is_cuda and codes.device == scales.device, "codes and scales: uint8, on one device")
        _need(codes.dim() == 2 and cols >= 1 and tuple(codes.shape) == (codes.shape[0], k // 2)
              and tuple(scales.shape) == (codes.shape[0], k // 32), "codes [rows][K / 2], scales [rows][K / 32], K = cols rounded up to 256")
        _need(codes.is_contiguous() and scales.is_contiguous(), "codes and scales: contiguous")
        self.rows, self.cols, self.device = codes.shape[0], int(cols), codes.device
        self._both, self._codes, self._scales = None, codes, scales

    @classmethod
    def empty(cls, rows, cols, device="cuda"):
        """Memory for a matrix: one allocation, the scales behind the codes."""
        groups = -(-int(cols) // 256)
        if rows < 0 or groups < 1:
            raise ValueError("rows >= 0, cols >= 1")
        q = cls.__new__(cls)
        q._both = torch.empty(rows * groups * 136, dtype=torch.uint8, device=device)
        q.rows, q.cols, q.device, q._codes, q._scales = rows, int(cols), q._both.device, None, None
        at = q._both.data_ptr()                             # memory of its own, which nobody else can move
        q._at = at, at + rows * groups * 128
        return q

    def __reduce__(self):                                   # a copy, or a pickle, is a matrix of its own memory
        return Mx4, (self.codes, self.scales, self.cols)

    @property
    def codes(self):
        if self._codes is None:
            n = self._both.numel() // 17 * 16
            self._codes = self._both[:n].view(self.rows, -(-self.cols // 256) * 128)
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            n = self._both.numel() // 17 * 16
            self._scales = self._both[n:].view(self.rows, -(-self.cols // 256) * 8)
        return self._scales

    def _pointers(self):
        if self._both is not None:
            return self._at
        return self._codes.data_ptr(), self._scales.data_ptr()


def mx4_quantize(x, by="rows", out=None):
    """x float32 / bfloat16 / float16 [rows][cols] -> Mx4 of the same shape; by="columns": the Mx4 of x transposed, its blocks
    running down the columns of x (a weight [k][n] as mx4_gemm takes it).  Rows, or columns, of x are contiguous."""
    if not (x.is_cuda and x.dim() == 2 and x.dtype in _DTYPES):
        raise ValueError("x: a matrix in float32, bfloat16 or float16 on the device")
    if by not in ("rows", "columns"):
        raise ValueError("by: 'rows' or 'columns'")
    if _tracked(x):
        raise ValueError("rounding to 4 bits has no gradient: detach x")
    down = by == "columns"
    ld = _row_stride(x)
    if ld is None:                                      # a transposed view: the other direction of its base
        x, down = x.t(), not down
        ld = _row_stride(x)
        _need(ld is not None, "x: rows or columns contiguous, not overlapping")
    rows, cols = (x.shape[1], x.shape[0]) if down else x.shape
    _need(cols >= 1, "rows of at least one element")
    if out is None:
        out = Mx4.empty(rows, cols, x.device)
    elif not (out.rows == rows and out.cols == cols and out.device == x.device):
        raise ValueError("out: of the result's shape, on x's device")
    if rows:
        _call("pahq_mx4_quantize", out.device, x.data_ptr(), _DTYPES[x.dtype], rows, cols, ld, 1 if down else 0, *out._pointers())
    return out


def _result(out, rows, cols, dtype, device):
    """(tensor, row stride): `out` checked, or a new one."""
    if out is None:
        if dtype not in _DTYPES:
            raise ValueError("dtype: float32, bfloat16 or float16")
        ld = cols or 1
        return torch.empty_strided((rows, cols), (ld, 1), dtype=dtype, device=device), ld
    ld = _row_stride(out) if out.dim() == 2 else None
    if not (out.shape == (rows, cols) and out.dtype in _DTYPES and out.device == device and ld is not None and not _tracked(out)):
        raise ValueError("out: [%d][%d] in float32, bfloat16 or float16, rows contiguous, on the operands' device, without a gradient" % (rows, cols))
    return out, ld


def mx4_dequantize(q, dtype=torch.float32, out=None):
    """The values of an Mx4, exact in float32 and bfloat16.  `out` brings its own dtype."""
    out, ld = _result(out, q.rows, q.cols, dtype, q.device)
    if q.rows:
        _call("pahq_mx4_dequantize", q.device, *q._pointers(), q.rows, q.cols, out.data_ptr(), _DTYPES[out.dtype], ld)
    return out


def mx4_gemm(a, w, bias=None, residual=None, dtype=torch.float32, out=None):
    """a Mx4 [m][k], w Mx4 [n][k] -> a w^T (+ bias float32 [n]) (+ residual [m][n] of the result's dtype; it may be `out`)."""
    m, n, device = a.rows, w.rows, a.device
    if a.cols != w.cols or device != w.device:
        raise ValueError("a [m][k] and w [n][k] on one device")
    out, ld = _result(out, m, n, dtype, device)
    bp = rp = None
    ld_res = ld
    if bias is not None:
        if not (bias.dtype == torch.float32 and bias.shape == (n,) and bias.device == device and bias.is_contiguous()
                and not _tracked(bias)):
            raise ValueError("bias: float32 [n], contiguous, without a gradient")
        bp = bias.data_ptr()
    if residual is not None:
        ld_res = _row_stride(residual) if residual.dim() == 2 else None
        if not (residual.shape == (m, n) and residual.dtype == out.dtype and residual.device == device and ld_res is not None
                and not _tracked(residual)):
            raise ValueError("residual: [m][n] of the result's dtype, rows contiguous, without a gradient")
        rp = residual.data_ptr()
    if m and n:
        _call("pahq_mx4_gemm", device, *a._pointers(), *w._pointers(), m, n, a.cols, bp, rp, ld_res, out.data_ptr(), _DTYPES[out.dtype], ld)
    return out


def rotary_table(rot_dim, theta=10000.0, scaling="none", factor=1.0, original=0.0, turns=(1.0, 32.0), device="cuda"):
    """The table `rotary` takes, int64 [rot_dim / 2] (bit patterns): frequencies theta^(-2 i / rot_dim), as they are
    ("none"), divided by `factor` ("linear"), of a stretched theta ("base"), or divided where a pair turns less than turns[0]
    times over `original` positions, kept from turns[1] times on and blended in between ("bands")."""
    return torch.from_numpy(rotary_entries(rot_dim, theta, scaling, factor, original, turns).view(np.int64)).to(device)


def _strides(t):
    tokens, heads, d = t.shape
    if t.is_contiguous():
        return heads * d, d
    st, sh, se = t.stride()
    if se != 1 and d > 1:
        raise ValueError("the elements of a head: contiguous")
    if heads <= 1:
        sh = d
    if tokens <= 1:
        st = max(heads - 1, 0) * sh + d
    return st, sh


def _rotary(x, positions, table, layout, magnitude, inverse, out):
    tokens, heads, d = x.shape
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    elif not (out.shape == x.shape and out.dtype == x.dtype and out.device == x.device):
        raise ValueError("out: of x's shape and dtype, on its device")
    if tokens and heads:
        st, sh = _strides(x)
        ot, oh = _strides(out)
        _call("pahq_rotary", x.device, x.data_ptr(), _DTYPES[x.dtype], tokens, heads, d, st, sh, positions.data_ptr(), table.data_ptr(), 2 * table.numel(),
              _LAYOUTS[layout], magnitude, 1 if inverse else 0, out.data_ptr(), ot, oh)
    return out


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, table, layout, magnitude, inverse):
        ctx.save_for_backward(positions, table)
        ctx.how = layout, magnitude, not inverse
        return _rotary(x, positions, table, layout, magnitude, inverse, None)

    @staticmethod
    def backward(ctx, grad):
        positions, table = ctx.saved_tensors
        if grad.shape[2] > 1 and grad.stride(2) != 1:       # an expanded or transposed gradient
            grad = grad.contiguous()
        return _Rotary.apply(grad, positions, table, *ctx.how), None, None, None, None, None


def rotary(x, positions, table, layout="half", magnitude=1.0, inverse=False, out=None):
    """Turns the first 2 * len(table) elements of every head of x [tokens][heads][d_head] by their tokens' positions (int64
    [tokens]); the rest of the head is copied.  layout: "half" (pairs i, i + rot / 2) or "interleaved" (pairs 2 i, 2 i + 1).
    inverse turns back (the gradient; x gets it by itself where autograd asks).  out may be x."""
    if not (x.is_cuda and x.dim() == 3 and x.dtype in _DTYPES):
        raise ValueError("x: [tokens][heads][d_head] in float32, bfloat16 or float16 on the device")
    tokens, _, d = x.shape
    if not (positions.dtype == torch.int64 and positions.shape == (tokens,) and positions.device == x.device
            and positions.is_contiguous()):
        raise ValueError("positions: int64 [tokens], contiguous, on x's device")
    if not (table.dtype == torch.int64 and table.dim() == 1 and table.device == x.device and 2 <= 2 * table.numel() <= d
            and table.is_contiguous()):
        raise ValueError("table: from rotary_table, on x's device, for at most d_head elements")
    if layout not in _LAYOUTS:
        raise ValueError("layout: 'half' or 'interleaved'")
    if _tracked(x) or out is not None and _tracked(out):
        _need(out is None, "out: not where a gradient is recorded")
        return _Rotary.apply(x, positions, table, layout, float(magnitude), bool(inverse))
    return _rotary(x, positions, table, layout, float(magnitude), bool(inverse), out)
