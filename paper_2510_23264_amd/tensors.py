"""The library's operators on device tensors (include/pahq.h, the section of that name) with torch tensors: matrices
in 4 microscaled bits and their product, rotary positions, and a paged cache of keys and values with the attention that reads it.

Every call enqueues on the current stream of its tensors' device (whichever device is current) and does not wait.  Results are
new tensors unless `out` is given.  Strided tensors are taken as they are where the C functions can walk them and refused
otherwise; nothing is copied behind the caller's back.  Arguments that do not fit raise ValueError, a refusal of the
library raises PahqError."""
from __future__ import annotations

import numpy as np
import torch
from torch.autograd import forward_ad

from .binding import lib, _chk, rotary_entries, tree_words

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_LAYOUTS = {"half": 0, "interleaved": 1}


class _Unloaded:
    """Stands for the extension (csrc/tensors_ext.cpp) until its first use, so that the package imports before it is built."""

    def __getattr__(self, name):
        global _ext
        lib()                                               # says so where nothing is built
        try:
            from . import _tensors
        except ImportError as e:
            raise RuntimeError("_tensors.so does not load: run `python -m paper_2510_23264_amd.build` first") from e
        _ext = _tensors
        return getattr(_tensors, name)


_ext = _Unloaded()


def _need(ok, what):
    if not ok:
        raise ValueError(what)


class Mx4:
    """A matrix [rows][cols] in 4 microscaled bits: `codes` uint8 [rows][K / 2] and `scales` uint8 [rows][K / 32], K = cols
    rounded up to 256, both contiguous on one device (the format is described in include/pahq.h)."""

    __slots__ = ("rows", "cols", "_both", "_codes", "_scales", "_at")

    def __init__(self, codes, scales, cols):
        k = -(-int(cols) // 256) * 256
        _need(codes.dtype == scales.dtype == torch.uint8 and codes.is_cuda and codes.device == scales.device, "codes and scales: uint8, on one device")
        _need(codes.dim() == 2 and cols >= 1 and tuple(codes.shape) == (codes.shape[0], k // 2)
              and tuple(scales.shape) == (codes.shape[0], k // 32), "codes [rows][K / 2], scales [rows][K / 32], K = cols rounded up to 256")
        _need(codes.is_contiguous() and scales.is_contiguous(), "codes and scales: contiguous")
        self.rows, self.cols = codes.shape[0], int(cols)
        self._both, self._codes, self._scales, self._at = None, codes, scales, None

    @classmethod
    def _of(cls, both, at):
        """One allocation, the scales behind the codes; `at`: addresses, sizes and device of memory that nobody else can move."""
        q = cls.__new__(cls)
        q.rows, q.cols = at[2], at[3]
        q._both, q._codes, q._scales, q._at = both, None, None, at
        return q

    @classmethod
    def empty(cls, rows, cols, device="cuda"):
        """Memory for a matrix."""
        groups = -(-int(cols) // 256)
        _need(rows >= 0 and groups >= 1, "rows >= 0, cols >= 1")
        both = torch.empty(rows * groups * 136, dtype=torch.uint8, device=device)
        _need(both.is_cuda, "a device")
        at = both.data_ptr()
        return cls._of(both, (at, at + rows * groups * 128, int(rows), int(cols), both.device.index))

    # a copy, shallow or deep, or a pickle, is a matrix of its own memory
    def __copy__(self):
        return Mx4(self.codes.clone(), self.scales.clone(), self.cols)

    def __reduce__(self):
        return Mx4, (self.codes, self.scales, self.cols)

    @property
    def device(self):
        return (self._codes if self._both is None else self._both).device

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

    def _where(self):
        if self._at is not None:
            return self._at
        return self._codes.data_ptr(), self._scales.data_ptr(), self.rows, self.cols, self._codes.device.index


def mx4_quantize(x, by="rows", out=None):
    """x float32 / bfloat16 / float16 [rows][cols] -> Mx4 of the same shape; by="columns": the Mx4 of x transposed, its blocks
    running down the columns of x (a weight [k][n] as mx4_gemm takes it).  Rows, or columns, of x are contiguous."""
    if by != "rows" and by != "columns":
        raise ValueError("by: 'rows' or 'columns'")
    got = _ext.mx4_quantize(x, by == "columns", None if out is None else out._where())
    if type(got) is int:
        _chk(got, "pahq_mx4_quantize")
    return Mx4._of(*got) if out is None else out


def mx4_dequantize(q, dtype=torch.float32, out=None):
    """The values of an Mx4, exact in float32 and bfloat16.  `out` brings its own dtype."""
    got = _ext.mx4_dequantize(q._where(), _DTYPES.get(dtype, -1), out)
    if type(got) is int:
        _chk(got, "pahq_mx4_dequantize")
    return got


def mx4_gemm(a, w, bias=None, residual=None, dtype=torch.float32, out=None):
    """a Mx4 [m][k], w Mx4 [n][k] -> a w^T (+ bias float32 [n]) (+ residual [m][n] of the result's dtype; it may be `out`)."""
    got = _ext.mx4_gemm(a._where(), w._where(), bias, residual, _DTYPES.get(dtype, -1), out)
    if type(got) is int:
        _chk(got, "pahq_mx4_gemm")
    return got


def rotary_table(rot_dim, theta=10000.0, scaling="none", factor=1.0, original=0.0, turns=(1.0, 32.0), device="cuda"):
    """The table `rotary` takes, int64 [rot_dim / 2] (bit patterns): frequencies theta^(-2 i / rot_dim), as they are
    ("none"), divided by `factor` ("linear"), of a stretched theta ("base"), or divided where a pair turns less than turns[0]
    times over `original` positions, kept from turns[1] times on and blended in between ("bands")."""
    return torch.from_numpy(rotary_entries(rot_dim, theta, scaling, factor, original, turns).view(np.int64)).to(device)


def _tangent(x):
    """Whether x has a forward-mode derivative to carry on, inside of a forward_ad.dual_level."""
    return torch._C._is_fwd_grad_enabled() and forward_ad.unpack_dual(x).tangent is not None


def _rotary(x, positions, table, layout, magnitude, inverse, out):
    got = _ext.rotary(x, positions, table, layout, magnitude, inverse, out)
    if type(got) is int:
        _chk(got, "pahq_rotary")
    return got


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, table, layout, magnitude, inverse):
        ctx.save_for_backward(positions, table)
        ctx.save_for_forward(positions, table)
        ctx.how = layout, magnitude, not inverse
        return _rotary(x, positions, table, layout, magnitude, inverse, None)

    @staticmethod
    def backward(ctx, grad):
        positions, table = ctx.saved_tensors
        if grad.shape[2] > 1 and grad.stride(2) != 1:       # an expanded or transposed gradient
            grad = grad.contiguous()
        return _Rotary.apply(grad, positions, table, *ctx.how), None, None, None, None, None

    @staticmethod
    def jvp(ctx, tangent, *_):                              # linear in x
        positions, table = ctx.saved_tensors
        layout, magnitude, back = ctx.how
        if tangent.shape[2] > 1 and tangent.stride(2) != 1:
            tangent = tangent.contiguous()
        return _Rotary.apply(tangent, positions, table, layout, magnitude, not back)


def rotary(x, positions, table, layout="half", magnitude=1.0, inverse=False, out=None):
    """Turns the first 2 * len(table) elements of every head of x [tokens][heads][d_head] by their tokens' positions (int64
    [tokens]); the rest of the head is copied.  layout: "half" (pairs i, i + rot / 2) or "interleaved" (pairs 2 i, 2 i + 1).
    inverse turns back (the gradient; x gets it by itself where autograd asks, and a tangent of x in forward mode is carried).  out
    may be x, except where a derivative is recorded."""
    if layout not in _LAYOUTS:
        raise ValueError("layout: 'half' or 'interleaved'")
    if torch.is_grad_enabled() and (x.requires_grad or out is not None and out.requires_grad) \
            or forward_ad._current_level >= 0 and _tangent(x):             # outside of a dual_level nothing has a tangent
        _need(out is None, "out: not where a gradient is recorded")
        return _Rotary.apply(x, positions, table, _LAYOUTS[layout], float(magnitude), bool(inverse))
    return _rotary(x, positions, table, _LAYOUTS[layout], magnitude, bool(inverse), out)


class KvCache:
    """A paged cache: `keys` and `values`, tensors [pages][heads][page_size][d_head] of float32, bfloat16 or float16 with the same strides, in any
    order in memory (permuted views, or the two halves of one tensor), elements of a row contiguous, everything else in whole 16
    bytes.  d_head: a multiple of 8 up to 256."""

    __slots__ = ("keys", "values")

    def __init__(self, keys, values):
        _need(keys.dim() == 4 and keys.shape == values.shape and keys.dtype == values.dtype and keys.dtype in _DTYPES
              and keys.device == values.device, "keys and values: [pages][heads][page_size][d_head] of one dtype, on one device")
        self.keys, self.values = keys, values

    @classmethod
    def empty(cls, pages, page_size, heads, d_head, dtype=torch.bfloat16, device="cuda"):
        """Memory for a cache: what it holds is not set."""
        both = torch.empty(2, pages, heads, page_size, d_head, dtype=dtype, device=device)
        return cls(both[0], both[1])


class KvBatch:
    """The sequences of a call, int32 tensors on the cache's device: `starts` [batch + 1], sequence b's new tokens being rows starts[b] to
    starts[b + 1] - 1 of the operators' rows; `lengths` [batch], the new tokens included, which are a sequence's last; `pages` [batch][width],
    each sequence's pages in order.  Row j of a sequence is row j % page_size of its page j // page_size.  The tensors are read when a
    call's kernels run, so a captured graph finds what they hold when it is replayed."""

    __slots__ = ("starts", "lengths", "pages")

    def __init__(self, starts, lengths, pages):
        _need(starts.dtype == lengths.dtype == pages.dtype == torch.int32 and starts.device == lengths.device == pages.device
              and starts.dim() == lengths.dim() == 1 and pages.dim() == 2 and len(starts) == len(lengths) + 1 and len(pages) == len(lengths),
              "starts [batch + 1], lengths [batch], pages [batch][width]: int32, on one device")
        self.starts, self.lengths, self.pages = starts, lengths, pages


def kv_append(cache, batch, k, v, positions=None, table=None, layout="half", magnitude=1.0, q=None, out=None):
    """Writes new tokens' rows into their sequences' pages: k [tokens][cache heads][d_head] turned as `rotary` turns it (table None: as it is),
    v as it is.  positions: int64 [tokens], or None for the tokens' rows in their sequences.  q [tokens][heads][d_head], if given, is
    turned the same way and returned (in `out`, which may be q).  Rows of tokens that belong to no sequence are not written."""
    if layout not in _LAYOUTS:
        raise ValueError("layout: 'half' or 'interleaved'")
    got = _ext.kv_append(cache.keys, cache.values, batch.starts, batch.lengths, batch.pages, k, v, positions, table, _LAYOUTS[layout], magnitude, q, out)
    if type(got) is int:
        _chk(got, "pahq_kv_append")
    return got


def tree_bits(parents, device="cuda"):
    """The masks `kv_attention` takes for a drafted tree, int64 [nodes][words] (bit patterns): every node sees itself and its ancestors.
    parents: each node's parent, which comes before it, -1 at a root.  Trees of a batch are joined below each other (torch.cat; of
    as many words)."""
    return torch.from_numpy(tree_words(parents).view(np.int64)).to(device)


def kv_attention(q, cache, batch, tree=None, scale=None, out=None):
    """Attention of the new tokens' queries q [tokens][heads][d_head] over their sequences' rows in the cache, whose heads go with heads / cache
    heads query heads each: a token sees the rows in front of the new ones, and of the new ones those up to itself, or those that
    its row of `tree` names (int64 [tokens][words], bit j % 64 of word j // 64 for new token j of its sequence).  scale: of the
    products, d_head ** -0.5 unless given.  A query that sees nothing gets zeros.  out may be q; rows of tokens that belong to no sequence are not written."""
    got = _ext.kv_attention(cache.keys, cache.values, batch.starts, batch.lengths, batch.pages, q, tree, scale, out)
    if type(got) is int:
        _chk(got, "pahq_kv_attention")
    return got


def kv_keep(cache, batch, paths, out=None):
    """Of each sequence's new tokens those that its row of paths (int32 [batch][depth], growing, -1 behind the last) names stay: their rows move
    together behind the ones in front of the new ones.  Returns the new lengths, int32 [batch] (in `out`, not the batch's own)."""
    got = _ext.kv_keep(cache.keys, cache.values, batch.starts, batch.lengths, batch.pages, paths, out)
    if type(got) is int:
        _chk(got, "pahq_kv_keep")
    return got
