"""Routed experts on torch tensors: routing, products in 8-bit blocks, and the products of the experts a row was routed to.

Every function checks what it is given, allocates its results and enqueues the library's kernels on the current stream of
the tensors' device; nothing is waited for and nothing is computed here.  Results have no history: tensors that want a gradient are refused
where gradients are recorded, and the *_backward calls form them.  Rows may be strided, their elements are consecutive.
Activations, logits and results are float32, bfloat16 or float16; what is kept in 8 bits is torch.float8_e4m3fn.

    rule = Rule(k=6, score=SIGMOID, scale=2.5)
    ids, weights = route(x @ centroids.t(), rule, bias=bias)         # the best six of the experts for every row
    y, kept = experts(x, ids, weights, w, train=True)                # w: quantize_weights(bf16 weights [E, N, K])
    d_x, d_w, d_weights = experts_backward(d_y, kept, w_turned)      # w_turned: quantize_weights(..., turned=True)
    d_logits = route_backward(logits, rule, ids, d_weights, bias=bias)
"""
from __future__ import annotations

from operator import attrgetter

import torch
from torch.autograd import forward_ad

from . import binding as B

SOFTMAX, SIGMOID = B.SCORE_SOFTMAX, B.SCORE_SIGMOID
BEST, BEST_TWO = B.GROUP_BEST, B.GROUP_BEST_TWO
BLOCK = 128
# Up to so many bytes of weights, an expert's counted for each row that goes to it, one launch without an order is faster than an order,
# products and sums, which take about 20 us more and read each expert's weights once.
DIRECT_BYTES = 128 << 20

_BYTES = (torch.float8_e4m3fn, torch.uint8)
_TYPES = {torch.float32: B.TYPE_F32, torch.bfloat16: B.TYPE_BF16, torch.float16: B.TYPE_F16}


def _type(dtype):
    code = _TYPES.get(dtype)
    if code is None:
        raise ValueError("float32, bfloat16 or float16 is wanted, not %s" % dtype)
    return code


# (the same numbers as torch.cuda.current_stream().cuda_stream and torch.cuda.current_device(), without the 3 us that their objects take)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream(t):
    if not t.is_cuda:
        raise ValueError("a tensor on the GPU is wanted; there is no CPU fallback")
    index = t.get_device()
    if index != _device():
        raise ValueError("the tensors are on %s, the current device is %d" % (t.device, _device()))
    return _raw_stream(index)


def _no_history(t, name):
    """Results have no history: what wants a gradient would lose it without a word.  (Under vmap and the transforms of torch.func tensors
    have no memory, which torch itself says.)"""
    if (t.requires_grad and torch.is_grad_enabled()) or (forward_ad._current_level >= 0 and forward_ad.unpack_dual(t).tangent is not None):
        raise ValueError("%s wants a gradient, which would be lost: detach it or call under torch.no_grad(), and use the *_backward calls" % name)


def _matrix(t, rows=None, cols=None, name="x"):
    """(type, rows, cols, stride) of a matrix whose rows are runs of consecutive elements."""
    if t.requires_grad or forward_ad._current_level >= 0:
        _no_history(t, name)
    shape = t.shape
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        raise ValueError("%s: a matrix%s is wanted, not %s" % (name, "" if rows is None and cols is None else " [%s, %s]" % (
            "..." if rows is None else rows, "..." if cols is None else cols), tuple(shape)))
    r, c = shape
    stride, inner = t.stride()
    if r <= 1:
        stride = c
    if (c > 1 and inner != 1) or stride < c:
        raise ValueError("%s: the elements of a row have to be consecutive and rows apart (strides %s)" % (name, t.stride()))
    return _type(t.dtype), r, c, stride


def _same_device(first, *others):
    index = first.get_device()                                      # (-1: the CPU)
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError("tensors on %s and %s" % (first.device, t.device))


def _flat(t, shape, dtype, name):
    if t.requires_grad or forward_ad._current_level >= 0:
        _no_history(t, name)
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s: a contiguous %s tensor %s is wanted, not %s %s" % (name, dtype, tuple(shape), t.dtype, tuple(t.shape)))


def _fixed(*names):
    """Attributes to be read: what the library is handed was made from them, and would not follow a change."""
    return (property(attrgetter("_" + name)) for name in names)


class Rule:
    """How experts are chosen: `k` of them by `score` (SOFTMAX, SIGMOID), out of the `kept` best of `groups` groups (judged by
    their BEST key or the sum of their BEST_TWO); with renormalize a row's weights add up to `scale`, else they are scores times `scale`."""
    __slots__ = ("_k", "_c")
    k, = _fixed("k")

    def __init__(self, k, score=SOFTMAX, groups=1, kept=1, group_by=BEST, renormalize=True, scale=1.0):
        self._k = k
        self._c = B.asgd_route_rule(k, score, groups, kept, group_by, int(renormalize), scale)


def route(logits, rule, bias=None):
    """(ids [T, k] int32, weights [T, k] float32) of the experts that rows of logits [T, E] are routed to; bias [E] float32 takes part in
    the choice alone.  -infinity in logits or bias takes an expert out; ids are -1 and weights 0 where none is left."""
    type, T, E, stride = _matrix(logits, name="logits")
    _same_device(logits, bias)
    if bias is not None:
        _flat(bias, (E,), torch.float32, "bias")
    s = _stream(logits)
    ids = logits.new_empty((T, rule._k), dtype=torch.int32)
    weights = torch.empty_like(ids, dtype=torch.float32)
    B.asgd_route(logits.data_ptr(), type, T, E, stride, None if bias is None else bias.data_ptr(), rule._c, ids.data_ptr(),
                 weights.data_ptr(), s)
    return ids, weights


def route_backward(logits, rule, ids, d_weights, bias=None):
    """The gradient of the logits [T, E], in their type, from that of route()'s weights; the choice is held fixed."""
    type, T, E, stride = _matrix(logits, name="logits")
    _same_device(logits, ids, d_weights, bias)
    _flat(ids, (T, rule._k), torch.int32, "ids")
    _flat(d_weights, (T, rule._k), torch.float32, "d_weights")
    if bias is not None:
        _flat(bias, (E,), torch.float32, "bias")
    s = _stream(logits)
    out = torch.empty((T, E), dtype=logits.dtype, device=logits.device)
    B.asgd_route_backward(logits.data_ptr(), type, T, E, stride, None if bias is None else bias.data_ptr(), rule._c, ids.data_ptr(),
                          d_weights.data_ptr(), out.data_ptr(), E, s)
    return out


class Plan:
    """The order in which experts take their rows (plan()): offsets [E + 1] (an expert's first place), blocks [E + 1] (its first block
    where each begins a new block of 128 places), slots [T * k] (the slot t * k + j at a place, -1: none), places [T * k] (the place of a
    slot, -1: none)."""
    __slots__ = ("_T", "_k", "_E", "_offsets", "_blocks", "_slots", "_places", "_c", "_memory")
    T, k, E, offsets, blocks, slots, places = _fixed("T", "k", "E", "offsets", "blocks", "slots", "places")

    def __init__(self, T, k, E, device):
        n = T * k
        self._T, self._k, self._E = T, k, E
        self._memory = m = torch.empty(2 * (E + 1) + 2 * n, dtype=torch.int32, device=device)
        self._offsets, self._blocks, self._slots, self._places = m[:E + 1], m[E + 1:2 * E + 2], m[2 * E + 2:2 * E + 2 + n], m[2 * E + 2 + n:]
        at = m.data_ptr()
        self._c = B.asgd_route_order(T, k, E, at, at + 4 * (E + 1), at + 8 * (E + 1), at + 8 * (E + 1) + 4 * n)

    def max_blocks(self):
        return B.asgd_route_max_blocks(self.T, self.k, self.E)


def plan(ids, experts):
    """The Plan of ids [T, k] (int32; what is outside 0 .. experts - 1 has no expert)."""
    if ids.dim() != 2:
        raise ValueError("ids: [T, k] is wanted, not %s" % (tuple(ids.shape),))
    _flat(ids, ids.shape, torch.int32, "ids")
    s = _stream(ids)
    p = Plan(ids.shape[0], ids.shape[1], experts, ids.device)
    size = B.asgd_route_plan_bytes(p._T, p._k, p._E)
    work = torch.empty(size, dtype=torch.uint8, device=ids.device) if size else None
    B.asgd_route_plan(ids.data_ptr(), p._c, None if work is None else work.data_ptr(), size, s)
    return p


class Blocks:
    """A matrix, or one for each expert, in 8-bit blocks: values [..., rows, 128 * ceil(cols / 128)] (float8_e4m3fn or uint8, zeros
    from `cols` on) times scales: squares [..., ceil(rows / 128), ceil(cols / 128)], or (squares=False) [ceil(cols / 128), rows]."""
    __slots__ = ("_values", "_scales", "_rows", "_cols", "_count", "_squares", "_c")
    values, scales, rows, cols, count, squares = _fixed("values", "scales", "rows", "cols", "count", "squares")

    def __init__(self, values, scales, cols, squares=True):
        kb, shape, dims = -(-cols // BLOCK), values.shape, values.dim()
        if values.dtype not in _BYTES or not (dims == 2 or (squares and dims == 3)) or shape[-1] != kb * BLOCK or not values.is_contiguous():
            raise ValueError("values: contiguous float8_e4m3fn or uint8 [%srows, %d] are wanted, not %s %s" % ("experts, " if squares else "", kb * BLOCK, values.dtype, tuple(shape)))
        rows, count = shape[-2], shape[0] if dims == 3 else 1
        _flat(scales, (kb, rows) if not squares else (-(-rows // BLOCK), kb) if dims == 2 else (count, -(-rows // BLOCK), kb), torch.float32, "scales")
        _same_device(values, scales)
        self._values, self._scales, self._rows, self._cols, self._squares, self._count = values, scales, rows, cols, squares, count
        self._c = B.asgd_blocks(values.data_ptr(), scales.data_ptr(), rows, cols, B.BLOCKS_SQUARES if squares else B.BLOCKS_ROWS, count, 0, 0)


def _sizes(x, turned, plan):
    """(rows, cols, blocks) of x in 8 bits."""
    rows, cols = x.shape
    if turned:
        out_rows, out_cols = cols, rows if plan is None else max(1, plan.max_blocks()) * BLOCK
    else:
        out_rows, out_cols = rows if plan is None else plan._T * plan._k, cols
    return out_rows, out_cols, -(-out_cols // BLOCK)


def _check_rows(x, plan, weights):
    """_matrix() of what is brought to 8 bits."""
    if weights is not None:
        if plan is None:
            raise ValueError("weights belong to the slots of a plan")
        _flat(weights, (plan._T, plan._k), torch.float32, "weights")
    if plan is not None:
        _same_device(x, plan._memory, weights)
    return _matrix(x, None if plan is None else plan._T)


class _Rows:
    """8-bit blocks of 1 x 128 that stay inside: one piece of memory, and the library's structure for it."""
    __slots__ = ("_memory", "_rows", "_cols", "_c")
    memory, rows, cols = _fixed("memory", "rows", "cols")

    def __init__(self, x, turned, plan):
        rows, cols, kb = _sizes(x, turned, plan)
        self._rows, self._cols = rows, cols
        n = rows * kb * BLOCK
        self._memory = torch.empty(n + 4 * kb * rows, dtype=torch.uint8, device=x.device)
        at = self._memory.data_ptr()
        self._c = B.asgd_blocks(at, at + n, rows, cols, B.BLOCKS_ROWS, 1, 0, 0)


def _quantized(x, turned=False, plan=None, weights=None):
    type, rows, cols, stride = _check_rows(x, plan, weights)
    s = _stream(x)
    out = _Rows(x, turned, plan)
    if rows:
        B.asgd_block_quantize(x.data_ptr(), type, rows, cols, stride, int(turned), None if plan is None else plan._c,
                              None if weights is None else weights.data_ptr(), out._c, s)
    return out


def _quantized_both(x, plan=None, weights=None):
    """(not turned, turned) from one reading of x."""
    type, rows, cols, stride = _check_rows(x, plan, weights)
    s = _stream(x)
    out, turned = _Rows(x, False, plan), _Rows(x, True, plan)
    if rows:
        B.asgd_block_quantize_both(x.data_ptr(), type, rows, cols, stride, None if plan is None else plan._c,
                                   None if weights is None else weights.data_ptr(), out._c, turned._c, s)
    return out, turned


def quantize(x, turned=False, plan=None, weights=None):
    """x [rows, cols] in 8-bit blocks of 1 x 128 (Blocks, squares=False), or with `turned` its transpose, blocks along x's rows.  With a
    plan x has a row for each of its T rows, and what is brought to 8 bits has one for each place: x's row of the place's slot, times the
    slot's weight (weights [T, k] float32) if given; turned, every expert's places begin a new block and the rest of its last one is zeros."""
    type, rows, cols, stride = _check_rows(x, plan, weights)
    s = _stream(x)
    out_rows, out_cols, kb = _sizes(x, turned, plan)
    out = Blocks(torch.empty((out_rows, kb * BLOCK), dtype=torch.float8_e4m3fn, device=x.device),
                 torch.empty((kb, out_rows), dtype=torch.float32, device=x.device), out_cols, squares=False)
    if rows:
        B.asgd_block_quantize(x.data_ptr(), type, rows, cols, stride, int(turned), None if plan is None else plan._c,
                              None if weights is None else weights.data_ptr(), out._c, s)
    return out


def quantize_weights(w, turned=False):
    """Weights [rows, cols] or [experts, rows, cols] in 8-bit squares of 128 x 128, or with `turned` their transposes (the same values:
    squares turn into squares), which the gradient of the activations takes."""
    if w.dim() not in (2, 3) or not w.is_contiguous() or w.numel() == 0:
        raise ValueError("weights: a contiguous [rows, cols] or [experts, rows, cols] is wanted, not %s" % (tuple(w.shape),))
    if w.requires_grad or forward_ad._current_level >= 0:
        _no_history(w, "weights")
    type, s, lead = _type(w.dtype), _stream(w), w.shape[:-2]
    rows, cols = w.shape[-2:]
    out_rows, out_cols = (cols, rows) if turned else (rows, cols)
    kb = -(-out_cols // BLOCK)
    out = Blocks(torch.empty((*lead, out_rows, kb * BLOCK), dtype=torch.float8_e4m3fn, device=w.device),
                 torch.empty((*lead, -(-out_rows // BLOCK), kb), dtype=torch.float32, device=w.device), out_cols)
    B.asgd_block_quantize(w.data_ptr(), type, rows, cols, cols, int(turned), None, None, out._c, s)
    return out


def _exact(dtype, exact):
    """Beside a rounding to bfloat16 what the 8-bit instruction drops does not show (4096^3: an error of 1.6602e-3 for 1.6599e-3, in half the
    time); beside one to float16 it does (2.096e-4 for 2.075e-4)."""
    return int(dtype != torch.bfloat16 if exact is None else exact)


def _product(a, b, dtype, plan, mode, exact, device):
    rows = a._rows if plan is None else plan._T * plan._k
    type, s = _type(dtype), _raw_stream(device.index)
    if a._cols == 0 and b._cols == 0:                                  # (a sum over nothing)
        return torch.zeros((rows, b._rows), dtype=dtype, device=device)
    out = torch.empty((rows, b._rows), dtype=dtype, device=device)
    if rows:
        B.asgd_block_product(a._c, b._c, mode, _exact(dtype, exact), None if plan is None else plan._c, out.data_ptr(), type, b._rows, s)
    return out


def _product_over(a, b, plan, dtype, exact, device):
    shape = (plan._E, a._rows, b._rows)
    if plan._T == 0:
        return torch.zeros(shape, dtype=dtype, device=device)
    out = torch.empty(shape, dtype=dtype, device=device)
    B.asgd_block_product(a._c, b._c, B.PRODUCT_OVER, _exact(dtype, exact), plan._c, out.data_ptr(), _type(dtype), b._rows, _raw_stream(device.index))
    return out


def product(a, b, dtype, plan=None, gather=False, exact=None):
    """a b^T in `dtype` of two Blocks of the same cols.  With a plan b has a matrix for each expert, and row p of the result is that of
    the place p with the matrix of its expert: a has a row for each place, or with `gather` one for each of the plan's T rows.  Rows at
    places that are not in use are left as they were allocated.  exact: the products of a block are summed in 32 bits, at half the rate, and
    not by the 8-bit matrix instruction, whose sums are off by some 2e-5 to 1e-4 of the result, more where large products cancel (None: in 32
    bits, but for bfloat16 results)."""
    _same_device(a._values, b._values, None if plan is None else plan._memory)
    _stream(a._values)
    return _product(a, b, dtype, plan, B.PRODUCT_ALL if plan is None else B.PRODUCT_GATHER if gather else B.PRODUCT_PLACES, exact, a._values.device)


def product_over(a, b, plan, dtype=torch.float32, exact=None):
    """[E, a.rows, b.rows]: for each expert a b^T over its own places alone; a and b are quantize(..., turned=True, plan=plan)."""
    _same_device(a._values, b._values, plan._memory)
    _stream(a._values)
    return _product_over(a, b, plan, dtype, exact, a._values.device)


def _raw(x):
    """x as an operand that the product brings to 8 bits itself."""
    type, rows, cols, stride = _matrix(x)
    return B.asgd_blocks(x.data_ptr(), None, rows, cols, B.BLOCKS_RAW, 1, type, stride)


def _product_of(x, w, dtype, plan=None, exact=None):
    """x, one row for each of the plan's T, times w."""
    rows = x.shape[0] if plan is None else plan._T * plan._k
    mode = B.PRODUCT_ALL if plan is None else B.PRODUCT_GATHER
    _same_device(x, w._values)
    # (few rows of an expert: bringing them to 8 bits again in each strip of its weights takes less than another launch)
    if not 0 < rows <= (B.PRODUCT_RAW_ROWS if plan is None else min(B.PRODUCT_RAW_SLOTS, 16 * plan._E)):
        return _product(_quantized(x), w, dtype, plan, mode, exact, x.device)
    raw, s = _raw(x), _stream(x)
    out = torch.empty((rows, w._rows), dtype=dtype, device=x.device)
    B.asgd_block_product(raw, w._c, mode, _exact(dtype, exact), None if plan is None else plan._c, out.data_ptr(), _type(dtype), w._rows, s)
    return out


def experts_sum(y, plan, dtype, weights=None):
    """[T, n] in `dtype`: the sum of each row's y [T * k, n] at the places of its slots, times weights [T, k] if given."""
    y_type, _, n, y_stride = _matrix(y, plan._T * plan._k, name="y")
    _same_device(y, plan._memory, weights)
    if weights is not None:
        _flat(weights, (plan._T, plan._k), torch.float32, "weights")
    s = _stream(y)
    out = torch.empty((plan._T, n), dtype=dtype, device=y.device)
    B.asgd_experts_sum(y.data_ptr(), y_type, n, y_stride, plan._c, None if weights is None else weights.data_ptr(), out.data_ptr(),
                       _type(dtype), n, s)
    return out


def experts_sum_backward(d_out, y, plan):
    """The gradient [T, k] float32 of experts_sum()'s weights from that of its result [T, n]."""
    y_type, _, n, y_stride = _matrix(y, plan._T * plan._k, name="y")
    type, _, _, stride = _matrix(d_out, plan._T, n, "d_out")
    _same_device(y, plan._memory, d_out)
    s = _stream(y)
    out = torch.empty((plan._T, plan._k), dtype=torch.float32, device=y.device)
    B.asgd_experts_sum_backward(d_out.data_ptr(), type, stride, y.data_ptr(), y_type, n, y_stride, plan._c, out.data_ptr(), s)
    return out


def _check_weights(x, w, experts=False):
    if not w._squares or (w._count != 1 and not experts):
        raise ValueError("weights in squares are wanted%s" % ("" if experts else ", one matrix of them"))
    if x.dim() != 2 or x.shape[1] != w._cols:
        raise ValueError("x: [rows, %d] is wanted, not %s" % (w._cols, tuple(x.shape)))


def linear(x, w, train=False, exact=None):
    """x [rows, K] times w^T, in x's type: x is brought to 8 bits on the way, w is quantize_weights() of [N, K].  train: (the result, what
    linear_backward() needs); the result is the same.  exact: as in product()."""
    _check_weights(x, w)
    if not train:
        return _product_of(x, w, x.dtype, exact=exact)
    _same_device(x, w._values)
    rows, turned = _quantized_both(x)
    return _product(rows, w, x.dtype, None, B.PRODUCT_ALL, exact, x.device), turned


def linear_backward(d_out, kept, w_turned, exact=None):
    """(d_x, in d_out's type, and d_w [N, K] float32) of linear(): from d_out [rows, N], what it kept, and the turned weights.  exact, as in
    product(), is for d_x; d_w is summed in 32 bits."""
    _check_weights(d_out, w_turned)
    if d_out.shape[0] != kept._cols or w_turned._rows != kept._rows:
        raise ValueError("d_out %s and the kept x [%d, %d] do not belong together" % (tuple(d_out.shape), kept._cols, kept._rows))
    _same_device(d_out, w_turned._values, kept._memory)
    rows, turned = _quantized_both(d_out)
    return (_product(rows, w_turned, d_out.dtype, None, B.PRODUCT_ALL, exact, d_out.device),
            _product(turned, kept, torch.float32, None, B.PRODUCT_ALL, True, d_out.device))


class Kept:
    """What experts_backward() needs of experts(): the plan, the weights themselves, not a copy, the experts' products y and x in 8 bits."""
    __slots__ = ("_plan", "_weights", "_y", "_x_turned", "_version")
    plan, weights, y, x_turned = _fixed("plan", "weights", "y", "x_turned")

    def __init__(self, plan, weights, y, x_turned):
        self._plan, self._weights, self._y, self._x_turned = plan, weights, y, x_turned
        self._version = self._written()

    def _written(self):
        """How often the weights were written to (tensors of inference mode do not count that)."""
        return None if self._weights.is_inference() else self._weights._version


def experts(x, ids, weights, w, train=False, exact=None):
    """[T, N] in x's type: for each row of x [T, K] the sum of its experts' products with it, weights [T, k] times w[ids] x, ids as route() gives
    them.  w is quantize_weights() of [E, N, K].  train: (the result, what experts_backward() needs).  The result is the same with it and
    without, but for up to 16 rows the order in which 32-bit sums are added.  exact: as in product(), but None is in 32 bits for every type,
    since the gradient of the weights, which is 32-bit, is formed from the products."""
    _check_weights(x, w, experts=True)
    _same_device(x, ids, weights, w._values)
    T = x.shape[0]
    if ids.dim() != 2 or ids.shape[0] != T:
        raise ValueError("ids: [%d, k] is wanted, not %s" % (T, tuple(ids.shape)))
    _flat(ids, ids.shape, torch.int32, "ids")
    _flat(weights, ids.shape, torch.float32, "weights")
    exact = exact is None or bool(exact)
    if not train and 0 < T <= B.PRODUCT_RAW_ROWS and ids.numel() * w._rows * w._cols <= DIRECT_BYTES:
        raw, s = _raw(x), _stream(x)
        out = torch.empty((T, w._rows), dtype=x.dtype, device=x.device)
        B.asgd_experts_direct(raw, ids.data_ptr(), weights.data_ptr(), ids.shape[1], w._c, int(exact), out.data_ptr(),
                              _type(x.dtype), w._rows, s)
        return out
    _matrix(x)
    order = plan(ids, w._count)
    # 32-bit until the sum: one rounding to the result's type
    y = _product_of(x, w, torch.float32, order, exact=exact)
    out = experts_sum(y, order, x.dtype, weights)
    return (out, Kept(order, weights, y, _quantized(x, turned=True, plan=order))) if train else out


def experts_backward(d_out, kept, w_turned, exact=None):
    """(d_x [T, K] in d_out's type, d_w [E, N, K] float32, d_weights [T, k] float32) of experts(), from d_out [T, N].  exact, as in
    product(), is for d_x; d_w is summed in 32 bits."""
    _check_weights(d_out, w_turned, experts=True)
    order, x_turned = kept._plan, kept._x_turned
    if d_out.shape[0] != order._T or w_turned._rows != x_turned._rows or w_turned._count != order._E:
        raise ValueError("d_out %s and weights of %d experts [%d, %d] do not belong to what was kept" % (
            tuple(d_out.shape), w_turned._count, w_turned._rows, w_turned._cols))
    if kept._version != kept._written():
        raise ValueError("the weights have changed since experts() was called with them")
    _same_device(d_out, w_turned._values, kept._y)
    d_weights = experts_sum_backward(d_out, kept._y, order)
    rows, turned = _quantized_both(d_out, order, kept._weights)
    d_rows = _product(rows, w_turned, torch.float32, order, B.PRODUCT_PLACES, _exact(d_out.dtype, exact), d_out.device)
    d_x = experts_sum(d_rows, order, d_out.dtype)
    return d_x, _product_over(turned, x_turned, order, torch.float32, True, d_out.device), d_weights
