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

import math

import torch
from torch.autograd import forward_ad

from . import binding as B
from . import experts as X

RUN = 256                        # columns that a row is laid out in whole runs of
SMALL = 32                       # columns that share a scale
# Up to so many weights, an expert's counted for each row that goes to it, and results, one launch without an order is faster than an order, products and sums,
# 27 us and more: 16 rows of six of 64 experts of 2048 x 2048 34 us for 34, 32 rows of two, at the first limit, 24 for 30; 512 rows of one of 512 x 512, at the second, 26
# for 35; 2048 of one of 256 x 64, beyond it, 52.
DIRECT_NUMBERS = 1 << 28
DIRECT_RESULTS = 1 << 18


def _runs(cols):
    return -(-cols // RUN)


class Micro:
    """A matrix, or one for each expert, in 4 bits: values [..., rows, 128 * ceil(cols / 256)] uint8, two e2m1 numbers a byte, the first in the low four
    bits, zeros from `cols` on; scales [..., rows, 8 * ceil(cols / 256)] uint8, 2^(byte - 127) for 32 columns each, 255: not a number."""
    __slots__ = ("_memory", "_values", "_scales", "_rows", "_cols", "_count", "_lead", "_c")
    rows, cols, count = X._fixed("rows", "cols", "count")

    def __init__(self, values, scales, cols):
        kf, shape = -(-cols // RUN), values.shape
        lead = shape[:-1]
        if values.dtype is not torch.uint8 or len(lead) not in (1, 2) or shape[-1] != kf * (RUN // 2) or not values.is_contiguous():
            raise ValueError("values: contiguous uint8 [..., rows, %d] are wanted, not %s %s" % (kf * (RUN // 2), values.dtype, tuple(shape)))
        if scales.dtype is not torch.uint8 or scales.shape != lead + (kf * (RUN // SMALL),) or not scales.is_contiguous():
            raise ValueError("scales: contiguous uint8 %s are wanted, not %s %s" % ((*lead, kf * (RUN // SMALL)), scales.dtype, tuple(scales.shape)))
        if values.get_device() != scales.get_device():
            raise ValueError("tensors on %s and %s" % (values.device, scales.device))
        self._memory, self._values, self._scales = values, values, scales
        self._set(lead, cols, values.data_ptr(), scales.data_ptr())

    def _set(self, lead, cols, values, scales):
        self._lead, self._rows, self._cols, self._count = lead, lead[-1], cols, lead[0] if len(lead) == 2 else 1
        self._c = B.asgd_blocks(values, scales, self._rows, cols, B.BLOCKS_FOURS, self._count, 0, 0)

    @classmethod
    def _empty(cls, lead, cols, like):
        """Room for one in one piece of memory (values and scales are made of it when they are asked for)."""
        self = cls.__new__(cls)
        n = math.prod(lead) * _runs(cols)
        self._memory = like.new_empty(n * (RUN // 2 + RUN // SMALL), dtype=torch.uint8)
        self._values = self._scales = None
        at = self._memory.data_ptr()
        self._set(lead, cols, at, at + n * (RUN // 2))
        return self

    @property
    def values(self):
        if self._values is None:
            n = self._memory.numel() // 17 * 16                        # (128 bytes of values, 8 of scales)
            self._values = self._memory[:n].view(*self._lead, -1) if n else self._memory.view(*self._lead, _runs(self._cols) * (RUN // 2))
        return self._values

    @property
    def scales(self):
        if self._scales is None:
            n = self._memory.numel() // 17 * 16
            self._scales = self._memory[n:].view(*self._lead, -1) if n else self._memory.view(*self._lead, _runs(self._cols) * (RUN // SMALL))
        return self._scales


def quantize(x):
    """x [rows, cols], or contiguous [experts, rows, cols], in 4 bits (Micro).  The scale of 32 columns is the power of two that takes their
    largest magnitude to at most 6, the largest number of the format, or to where it is cut to it (below 7; below 8 from 1.75 * 2^127 on, where the
    next scale's numbers would pass float32); a block with something that is not a finite number is not a number."""
    if x.dim() == 3:
        if not x.is_contiguous() or x.numel() == 0:
            raise ValueError("x: a contiguous [experts, rows, cols] is wanted, not %s" % (tuple(x.shape),))
        if x.requires_grad or forward_ad._current_level >= 0:
            X._no_history(x, "x")
        lead, (rows, cols) = x.shape[:2], x.shape[1:]
        type, stride = X._type(x.dtype), cols
    else:
        type, rows, cols, stride = X._matrix(x)
        lead = (rows,)
    s = X._stream(x)
    out = Micro._empty(lead, cols, x)
    if rows:
        B.asgd_block_quantize(x.data_ptr(), type, rows, cols, stride, 0, None, None, out._c, s)
    return out


def expand(m, dtype=torch.float32):
    """The values that m stands for, [..., rows, cols] in `dtype`."""
    type, s = X._type(dtype), X._stream(m._memory)
    out = m._memory.new_empty((*m._lead, m._cols), dtype=dtype)
    if out.numel():
        B.asgd_block_expand(m._c, out.data_ptr(), type, m._cols, s)
    return out


def product(a, b, dtype, plan=None, gather=False):
    """a b^T in `dtype` of two Micro of the same cols.  With a plan b has a matrix for each expert, and row p of the result is that of
    the place p with the matrix of its expert: a has a row for each place, or with `gather` one for each of the plan's T rows.  Rows at
    places that are not in use are left as they were allocated.  Products are summed in 32 bits."""
    X._same_device(a._memory, b._memory, None if plan is None else plan._memory)
    type, s = X._type(dtype), X._stream(a._memory)
    rows = a._rows if plan is None else plan._T * plan._k
    out = a._memory.new_empty((rows, b._rows), dtype=dtype)
    if rows:
        B.asgd_block_product(a._c, b._c, B.PRODUCT_ALL if plan is None else B.PRODUCT_GATHER if gather else B.PRODUCT_PLACES, 1,
                             None if plan is None else plan._c, out.data_ptr(), type, b._rows, s)
    return out


def _check(x, w, experts=False):
    if type(w) is not Micro or (w._count != 1 and not experts):
        raise ValueError("weights in 4 bits are wanted%s" % ("" if experts else ", one matrix of them"))
    shape = x.shape
    if len(shape) != 2 or shape[1] != w._cols:
        raise ValueError("x: [rows, %d] is wanted, not %s" % (w._cols, tuple(shape)))
    return shape[0]


def linear(x, w):
    """x [rows, K] times w^T, in x's type: x is brought to 4 bits on the way, w is quantize() of [N, K]."""
    rows = _check(x, w)
    if x.get_device() != w._memory.get_device():
        X._same_device(x, w._memory)
    raw = X._raw(x)
    s, out, type = X._stream(x), x.new_empty((rows, w._rows)), raw.type
    # (few rows: bringing them to 4 bits again in each strip of the weights takes less than another launch)
    if rows > B.PRODUCT_RAW_ROWS:
        n = rows * _runs(w._cols)
        memory = x.new_empty(n * (RUN // 2 + RUN // SMALL), dtype=torch.uint8)
        at = memory.data_ptr()
        small = B.asgd_blocks(at, at + n * (RUN // 2), rows, w._cols, B.BLOCKS_FOURS, 1, 0, 0)
        B.asgd_block_quantize(raw.values, type, rows, w._cols, raw.stride, 0, None, None, small, s)
        raw = small
    if rows:
        B.asgd_block_product(raw, w._c, B.PRODUCT_ALL, 1, None, out.data_ptr(), type, w._rows, s)
    return out


def experts(x, ids, weights, w):
    """[T, N] in x's type: for each row of x [T, K] the sum of its experts' products with it, weights [T, k] times w[ids] x, ids as
    experts.route() gives them (what is outside 0 .. E - 1 has no expert).  w is quantize() of [E, N, K]; x is brought to 4 bits on the way."""
    T = _check(x, w, experts=True)
    X._same_device(x, ids, weights, w._memory)
    if ids.dim() != 2 or ids.shape[0] != T:
        raise ValueError("ids: [%d, k] is wanted, not %s" % (T, tuple(ids.shape)))
    X._flat(ids, ids.shape, torch.int32, "ids")
    X._flat(weights, ids.shape, torch.float32, "weights")
    raw = X._raw(x)
    s, slots = X._stream(x), ids.numel()
    if 0 < T <= B.PRODUCT_RAW_SLOTS and slots * w._rows * w._cols <= DIRECT_NUMBERS and T * w._rows <= DIRECT_RESULTS:
        out = x.new_empty((T, w._rows))
        B.asgd_experts_direct(raw, ids.data_ptr(), weights.data_ptr(), ids.shape[1], w._c, 1, out.data_ptr(), raw.type, w._rows, s)
        return out
    order = X.plan(ids, w._count)
    # 32-bit until the sum: one rounding to the result's type.  (Few rows of an expert are brought to 4 bits inside the product.)
    if 0 < slots <= min(B.PRODUCT_RAW_SLOTS, 16 * w._count):
        y = torch.empty((slots, w._rows), dtype=torch.float32, device=x.device)
        B.asgd_block_product(raw, w._c, B.PRODUCT_GATHER, 1, order._c, y.data_ptr(), B.TYPE_F32, w._rows, s)
    else:
        y = product(quantize(x), w, torch.float32, order, gather=True)
    return X.experts_sum(y, order, x.dtype, weights)
