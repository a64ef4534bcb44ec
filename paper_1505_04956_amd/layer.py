"""A whole layer of experts for a few rows on torch tensors: routing, both matrices of every chosen expert with a gated activation
between them, and each row's sum, in one call.

    rule = experts.Rule(k=6)
    up, down = experts.quantize_weights(w_up), experts.quantize_weights(w_down)       # [E, 2 * H, D] and [E, N, H]; or micro.quantize()
    y, ids, weights = layer(x, x @ centroids.t(), rule, up, down)

For prompts and for training there are the calls that it stands for: experts.route(), plan() and product().
"""
from __future__ import annotations

from functools import lru_cache

import torch

from . import binding as B
from . import experts as X
from . import micro as M

SILU, GELU = B.ACTIVATION_SILU, B.ACTIVATION_GELU
ROWS = B.PRODUCT_RAW_ROWS        # that a call takes at most


@lru_cache(maxsize=256)
def _scratch_bytes(T, k, E, D, H):
    return B.asgd_experts_layer_bytes(T, k, E, D, H)


def layer(x, logits, rule, up, down, bias=None, activation=SILU):
    """(y [T, N] in x's type, ids [T, k] int32, weights [T, k] float32) for at most 16 rows x [T, D].  ids and weights are those of
    experts.route(logits [T, E], rule, bias).  up has 2 * H rows of D columns for each expert, the gate's H first: u = up[e] x; h = f(u[:H]) * u[H:] with
    f(g) = g / (1 + exp(-g)) (SILU) or g / 2 * (1 + erf(g / sqrt(2))) (GELU); y is the sum of weights times down[e] h, down N rows of H columns for each
    expert, zeros for a row that has no expert.  up and down are both experts.quantize_weights() (x and h are brought to 8 bits on the way) or both
    micro.quantize() (to 4 bits); h and all sums are 32-bit."""
    if type(up) is not type(down) or not isinstance(up, (X.Blocks, M.Micro)) or (isinstance(up, X.Blocks) and not (up._squares and down._squares)):
        raise ValueError("up and down: both experts.quantize_weights() or both micro.quantize() are wanted")
    E = up._count
    if down._count != E or up._rows != 2 * down._cols:
        raise ValueError("up, %d experts [%d, %d], and down, %d [%d, %d], do not belong together" % (
            E, up._rows, up._cols, down._count, down._rows, down._cols))
    X._same_device(x, logits, *((up._memory, down._memory) if isinstance(up, M.Micro) else (up._values, down._values)), bias)
    raw = X._raw(x)
    T = raw.rows
    if x.shape[1] != up._cols or T > ROWS:
        raise ValueError("x: at most %d rows of %d are wanted, not %s" % (ROWS, up._cols, tuple(x.shape)))
    type_of_logits, _, _, stride = X._matrix(logits, T, E, "logits")
    if bias is not None:
        X._flat(bias, (E,), torch.float32, "bias")
    s, k = X._stream(x), rule._k
    y = x.new_empty((T, down._rows))
    ids = x.new_empty((T, k), dtype=torch.int32)
    weights = x.new_empty((T, k), dtype=torch.float32)
    if not T:
        return y, ids, weights
    size = _scratch_bytes(T, k, E, up._cols, down._cols)
    work = x.new_empty(size, dtype=torch.uint8)
    B.asgd_experts_layer(raw, logits.data_ptr(), type_of_logits, stride, None if bias is None else bias.data_ptr(), rule._c, up._c, down._c,
                         activation, ids.data_ptr(), weights.data_ptr(), y.data_ptr(), raw.type, down._rows, work.data_ptr(), size, s)
    return y, ids, weights
