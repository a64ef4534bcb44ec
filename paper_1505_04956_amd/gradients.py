"""The norm of many gradients together, and clipping by it, on torch tensors.

    d_x, d_w, d_weights = experts.experts_backward(d_y, kept, w_turned)
    norm = clip([d_w, d_shared, d_centroids], 1.0)           # in place; the norm before

Tensors are contiguous, float32, bfloat16 or float16 in any mixture, on one device.  The kernels are enqueued on its current stream, nothing is waited
for: the norm is a tensor, and what it decides is decided on the GPU.
"""
from __future__ import annotations

from array import array
from functools import lru_cache

import torch
from torch.autograd import forward_ad
from torch.autograd.graph import increment_version

from . import binding as B
from . import experts as X


def _spans(tensors, index, name):
    """(ptr, n, type) of each, one after the other, for the library."""
    spans, types, dual = [], X._TYPES, forward_ad._current_level >= 0
    for t in tensors:
        if t.requires_grad or dual:
            X._no_history(t, name)
        if t.get_device() != index:
            raise ValueError("tensors on %s and %s" % (tensors[0].device, t.device))
        if not t.is_contiguous():
            raise ValueError("%s: contiguous tensors are wanted, not %s with strides %s" % (name, tuple(t.shape), t.stride()))
        code = types.get(t.dtype)
        spans += (t.data_ptr(), t.numel(), X._type(t.dtype) if code is None else code)
    return array("q", spans)


def _prepare(tensors):
    tensors = list(tensors)
    if not tensors:
        raise ValueError("no tensors")
    return tensors, _spans(tensors, tensors[0].get_device(), "gradients")


@lru_cache(maxsize=64)
def _scratch_bytes(count):
    return B.asgd_gradient_bytes(count)


def _memory(count, like):
    size = _scratch_bytes(count)
    return like.new_empty((), dtype=torch.float32), like.new_empty(size, dtype=torch.uint8), size


def norm(tensors):
    """The square root of the sum of the squares of all elements of all tensors, a float32 tensor without dimensions.  Squares are added
    in 64 bits: it is infinite only where an element is, or the norm is beyond float32.  The same tensors give the same bits."""
    tensors, spans = _prepare(tensors)
    s = X._stream(tensors[0])
    out, work, size = _memory(len(tensors), tensors[0])
    B.asgd_gradient_norm(spans.buffer_info()[0], len(tensors), out.data_ptr(), work.data_ptr(), size, s)
    return out


def clip(tensors, limit, out=None):
    """Multiplies all elements by limit / norm(tensors) where the norm is larger than limit, and returns the norm, a float32 tensor without dimensions.  In
    place, or into `out`, tensors of as many elements and of any of the three types, in the same order: each is its gradient itself or shares no
    memory with any other (gradients that are only read may).  What is written counts as modified for autograd, as by an operation of torch in place, whether or not the norm is larger.  A norm that is not a number makes all elements not a number; an infinite one makes the finite elements zeros."""
    limit = float(limit)
    if not limit >= 0.0:
        raise ValueError("limit: a number from 0 on is wanted, not %r" % limit)
    tensors, spans = _prepare(tensors)
    to = None
    if out is not None:
        out = list(out)
        to = _spans(out, tensors[0].get_device(), "out")
        if to[1::3] != spans[1::3]:
            raise ValueError("out: a tensor of as many elements for each gradient is wanted")
    s = X._stream(tensors[0])
    result, work, size = _memory(len(tensors), tensors[0])
    B.asgd_gradient_clip(spans.buffer_info()[0], None if to is None else to.buffer_info()[0], len(tensors), limit, result.data_ptr(),
                         work.data_ptr(), size, s)
    increment_version(tensors if out is None else out)      # (what is written through an address autograd does not see; 1.4 us for three tensors, 32 for 400)
    return result
