"""Matrices in 4-bit floating point on torch tensors: two values a byte with a power of two as scale for each 32 columns, and their products.

What experts.py has in 8 bits for products that are not trained: a quarter of the bytes of 16-bit weights, at up to twice the 8-bit rate.  Every
function checks what it is given, allocates its results and enqueues the library's kernels on the current stream of the tensors'
device.  Results have no history.  Rows may be strided, their elements are consecutive; activations and results are float32,
bfloat16 or float16.

    w = quantize(weights)                                   # [N, K] or [E, N, K]
    y = linear(x, w)                                        # x [rows, K], brought to 4 bits on the way
    y = experts(x, ids, weights, w)                         # ids and weights as experts.route() gives them
"""
from __future__ import annotations

import torch
from torch.autograd import forward_ad

from . import binding as B
from . import experts as X

RUN = 256                        # columns that a row is laid out in whole runs of
SMALL = 32                       # columns that share a scale


def _runs(cols):
    return -(-cols // RUN)


class Micro:
    """A matrix, or one for each expert, in 4 bits: values [..., rows, 128 * ceil(cols / 256)] uint8, two e2m1 numbers a byte, the first in the low four
    bits, zeros from `cols` on; scales [..., rows, 8 * ceil(cols / 256)] uint8, 2^(byte - 127) for 32 columns each, 255: not a number."""
    __slots__ = ("_values", "_scales", "_rows", "_cols", "_count", "_c")
    values, scales, rows, cols, count = X._fixed("values", "scales", "rows", "cols", "count")

    def __init__(self, values, scales, cols):
        kf, shape, dims = _runs(cols), values.shape, values.dim()
        if values.dtype is not torch.uint8 or dims not in (2, 3) or shape[-1] != kf * (RUN // 2) or not values.is_contiguous():
            raise ValueError("values: contiguous uint8 [..., rows, %d] are wanted, not %s %s" % (kf * (RUN // 2), values.dtype, tuple(shape)))
        X._flat(scales, (*shape[:-1], kf * (RUN // SMALL)), torch.uint8, "scales")
        X._same_device(values, scales)
        self._set(values, scales, cols)

    def _set(self, values, scales, cols):
        shape = values.shape
        self._values, self._scales, self._cols = values, scales, cols
        self._rows, self._count = shape[-2], shape[0] if len(shape) == 3 else 1
        self._c = B.asgd_blocks(values.data_ptr(), scales.data_ptr(), self._rows, cols, B.BLOCKS_FOURS, self._count, 0, 0)


def quantize(x):
    """x [rows, cols], or contiguous [experts, rows, cols], in 4 bits (Micro).  The scale of 32 columns is the power of two that takes their
    largest magnitude to at most 6, the largest number of the format, or to where it is cut to it (below 7); a block with something that is not a finite number is not a number."""
    if x.dim() == 3:
        if not x.is_contiguous() or x.numel() == 0:
            raise ValueError("x: a contiguous [experts, rows, cols] is wanted, not %s" % (tuple(x.shape),))
        if x.requires_grad or forward_ad._current_level >= 0:
            X._no_history(x, "x")
        lead, rows, cols = x.shape[:1], *x.shape[1:]
        type, stride = X._type(x.dtype), cols
    else:
        type, rows, cols, stride = X._matrix(x)
        lead = ()
    s = X._stream(x)
    out = Micro.__new__(Micro)
    out._set(torch.empty((*lead, rows, _runs(cols) * (RUN // 2)), dtype=torch.uint8, device=x.device),
             torch.empty((*lead, rows, _runs(cols) * (RUN // SMALL)), dtype=torch.uint8, device=x.device), cols)
    if rows:
        B.asgd_block_quantize(x.data_ptr(), type, rows, cols, stride, 0, None, None, out._c, s)
    return out


def expand(m, dtype=torch.float32):
    """The values that m stands for, [..., rows, cols] in `dtype`."""
    type, s = X._type(dtype), X._stream(m._values)
    out = torch.empty((*m._values.shape[:-1], m._cols), dtype=dtype, device=m._values.device)
    if out.numel():
        B.asgd_block_expand(m._c, out.data_ptr(), type, m._cols, s)
    return out


def _product(a, rows, w, dtype, plan, mode, out_rows, device):
    type, s = X._type(dtype), X._raw_stream(device.index)
    out = torch.empty((out_rows, w._rows), dtype=dtype, device=device)
    if out_rows:
        B.asgd_block_product(a, w._c, mode, 1, None if plan is None else plan._c, out.data_ptr(), type, w._rows, s)
    return out


def product(a, b, dtype, plan=None, gather=False):
    """a b^T in `dtype` of two Micro of the same cols.  With a plan b has a matrix for each expert, and row p of the result is that of
    the place p with the matrix of its expert: a has a row for each place, or with `gather` one for each of the plan's T rows.  Rows at
    places that are not in use are left as they were allocated.  Products are summed in 32 bits."""
    X._same_device(a._values, b._values, None if plan is None else plan._memory)
    X._stream(a._values)
    return _product(a._c, a._rows, b, dtype, plan, B.PRODUCT_ALL if plan is None else B.PRODUCT_GATHER if gather else B.PRODUCT_PLACES,
                    a._rows if plan is None else plan._T * plan._k, a._values.device)


def _product_of(x, w, dtype, plan=None):
    """x, one row for each of the plan's T, times w."""
    rows = x.shape[0] if plan is None else plan._T * plan._k
    mode = B.PRODUCT_ALL if plan is None else B.PRODUCT_GATHER
    # (few rows of an expert: bringing them to 4 bits again in each strip of its weights takes less than another launch)
    if 0 < rows <= (B.PRODUCT_RAW_ROWS if plan is None else min(B.PRODUCT_RAW_SLOTS, 16 * plan._E)):
        raw = X._raw(x)
        X._stream(x)
    else:
        small = quantize(x)
        raw = small._c
    return _product(raw, x.shape[0], w, dtype, plan, mode, rows, x.device)


def _check(x, w, experts=False):
    if not isinstance(w, Micro) or (w._count != 1 and not experts):
        raise ValueError("weights in 4 bits are wanted%s" % ("" if experts else ", one matrix of them"))
    if x.dim() != 2 or x.shape[1] != w._cols:
        raise ValueError("x: [rows, %d] is wanted, not %s" % (w._cols, tuple(x.shape)))


def linear(x, w):
    """x [rows, K] times w^T, in x's type: x is brought to 4 bits on the way, w is quantize() of [N, K]."""
    _check(x, w)
    X._same_device(x, w._values)
    return _product_of(x, w, x.dtype)


def experts(x, ids, weights, w):
    """[T, N] in x's type: for each row of x [T, K] the sum of its experts' products with it, weights [T, k] times w[ids] x, ids as
    experts.route() gives them (what is outside 0 .. E - 1 has no expert).  w is quantize() of [E, N, K]; x is brought to 4 bits on the way."""
    _check(x, w, experts=True)
    X._same_device(x, ids, weights, w._values)
    T = x.shape[0]
    if ids.dim() != 2 or ids.shape[0] != T:
        raise ValueError("ids: [%d, k] is wanted, not %s" % (T, tuple(ids.shape)))
    X._flat(ids, ids.shape, torch.int32, "ids")
    X._flat(weights, ids.shape, torch.float32, "weights")
    if 0 < T <= B.PRODUCT_RAW_ROWS and ids.numel() * w._rows * w._cols <= 2 * X.DIRECT_BYTES:
        raw, s = X._raw(x), X._stream(x)
        out = torch.empty((T, w._rows), dtype=x.dtype, device=x.device)
        B.asgd_experts_direct(raw, ids.data_ptr(), weights.data_ptr(), ids.shape[1], w._c, 1, out.data_ptr(), X._type(x.dtype), w._rows, s)
        return out
    X._matrix(x)
    order = X.plan(ids, w._count)
    return X.experts_sum(_product_of(x, w, torch.float32, order), order, x.dtype, weights)
