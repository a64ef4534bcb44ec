"""What the routed experts refuse: the C entry points before anything is enqueued, the tensor calls before that.  No GPU is needed."""
import ctypes as C

import pytest
import torch

from paper_1505_04956_amd import binding as B
from paper_1505_04956_amd import experts as X
from tests import experts_rules as R

P = 1 << 20                                       # stands for a device pointer: these calls do not get as far as using it


def rule(**over):
    base = dict(k=2, score=B.SCORE_SOFTMAX, groups=1, kept=1, group_by=B.GROUP_BEST, renormalize=1, scale=1.0)
    base.update(over)
    return B.asgd_route_rule(*(base[f] for f, _ in B.asgd_route_rule._fields_))


def route(r=None, logits=P, type=0, T=4, E=8, stride=8, bias=None, ids=P, weights=P):
    r = r or rule()
    return B.lib().asgd_route(logits, type, T, E, stride, bias, C.addressof(r), ids, weights, None)


@pytest.mark.parametrize("over", [dict(k=0), dict(k=9), dict(k=65), dict(score=2), dict(groups=0), dict(groups=3), dict(groups=65), dict(kept=0),
                                  dict(kept=2), dict(groups=4, kept=1, k=3), dict(group_by=2), dict(groups=8, kept=8, group_by=1),
                                  dict(renormalize=2), dict(scale=float("inf")), dict(scale=float("nan"))])
def test_rules_that_are_refused(over):
    assert route(rule(**over)) == B.EINVAL
    r = rule(**over)
    assert B.lib().asgd_route_backward(P, 0, 4, 8, 8, None, C.addressof(r), P, P, P, 8, None) == B.EINVAL


@pytest.mark.parametrize("over", [dict(logits=None), dict(logits=P + 2), dict(type=3), dict(type=-1), dict(T=-1), dict(E=0), dict(E=1025), dict(stride=7),
                                  dict(stride=-8), dict(ids=None), dict(weights=None), dict(weights=P + 1), dict(bias=P + 2)])
def test_routes_that_are_refused(over):
    assert route(**over) == B.EINVAL


def test_nothing_to_do_is_no_error():
    assert route(T=0, logits=None, ids=None, weights=None) == B.OK
    assert B.lib().asgd_route(P, 0, 4, 8, 8, None, None, P, P, None) == B.EINVAL


def order(**over):
    base = dict(T=4, k=2, E=3, offsets=P, blocks=P, slots=P, places=P)
    base.update(over)
    return B.asgd_route_order(*(base[f] for f, _ in B.asgd_route_order._fields_))


@pytest.mark.parametrize("over", [dict(T=-1), dict(k=0), dict(k=65), dict(E=0), dict(E=1025), dict(T=1 << 30), dict(offsets=None), dict(blocks=None),
                                  dict(slots=None), dict(places=P + 2)])
def test_orders_that_are_refused(over):
    o = order(**over)
    assert B.lib().asgd_route_plan(P, C.addressof(o), None, 0, None) == B.EINVAL
    assert B.lib().asgd_experts_sum(P, 0, 8, 8, C.addressof(o), None, P, 0, 8, None) == B.EINVAL


def test_scratch_of_the_order():
    assert B.asgd_route_plan_bytes(4, 2, 3) == 0
    need = B.asgd_route_plan_bytes(100_000, 8, 256)
    assert need > 0
    o = order(T=100_000, k=8, E=256)
    for work, size in ((None, need), (P, need - 1), (P + 4, need)):
        assert B.lib().asgd_route_plan(P, C.addressof(o), work, size, None) == B.EINVAL
    assert B.asgd_route_max_blocks(0, 4, 8) == 0 and B.asgd_route_max_blocks(1, 4, 8) == 4 and B.asgd_route_max_blocks(1000, 4, 8) == 31 + 8


def blocks(**over):
    base = dict(values=P, scales=P, rows=8, cols=200, form=B.BLOCKS_ROWS, count=1, type=0, stride=0)
    base.update(over)
    return B.asgd_blocks(*(base[f] for f, _ in B.asgd_blocks._fields_))


def quantize(out, x=P, type=1, rows=8, cols=200, stride=200, turned=0, o=None, weights=None):
    return B.lib().asgd_block_quantize(x, type, rows, cols, stride, turned, None if o is None else C.addressof(o), weights, C.addressof(out), None)


def test_bringing_to_eight_bits_that_is_refused():
    for out in (blocks(values=None), blocks(scales=None), blocks(values=P + 8), blocks(rows=9), blocks(cols=199), blocks(form=3), blocks(form=B.BLOCKS_RAW, type=1, stride=200),
                blocks(count=2), blocks(count=0)):
        assert quantize(out) == B.EINVAL
    for over in (dict(x=None), dict(x=P + 1), dict(type=4), dict(rows=-1), dict(cols=0), dict(stride=199), dict(turned=2), dict(weights=P), dict(turned=1)):
        assert quantize(blocks(), **over) == B.EINVAL
    o = order(T=8, k=2, E=3)
    assert quantize(blocks(rows=15), o=o) == B.EINVAL                                    # T * k rows
    assert quantize(blocks(rows=16, form=B.BLOCKS_SQUARES), o=o) == B.EINVAL
    assert quantize(blocks(rows=16), rows=7, o=o) == B.EINVAL
    assert quantize(blocks(rows=200, cols=128), turned=1, o=o) == B.EINVAL               # 3 blocks


def test_both_ways_that_are_refused():
    def go(out=None, turned=None, x=P, type=1, rows=8, cols=200, stride=200, o=None, weights=None):
        out, turned = out or blocks(), turned or blocks(rows=200, cols=8)
        return B.lib().asgd_block_quantize_both(x, type, rows, cols, stride, None if o is None else C.addressof(o), weights, C.addressof(out), C.addressof(turned), None)
    for over in (dict(out=blocks(rows=9)), dict(out=blocks(form=B.BLOCKS_SQUARES)), dict(turned=blocks(rows=200, cols=9)), dict(turned=blocks(rows=199, cols=8)),
                 dict(turned=blocks(rows=200, cols=8, values=None)), dict(x=None), dict(type=7), dict(rows=-1), dict(stride=199), dict(weights=P), dict(o=order(T=8, k=2, E=3))):
        assert go(**over) == B.EINVAL


def product(a, b, mode=B.PRODUCT_ALL, exact=0, o=None, out=P, type=0, stride=8):
    return B.lib().asgd_block_product(C.addressof(a), C.addressof(b), mode, exact, None if o is None else C.addressof(o), out, type, stride, None)


def test_products_that_are_refused():
    a, b, sq = blocks(), blocks(), blocks(form=B.BLOCKS_SQUARES)
    for x, y in ((blocks(cols=199), b), (sq, b), (a, blocks(form=B.BLOCKS_RAW, stride=200)), (a, blocks(form=B.BLOCKS_SQUARES, count=2)), (blocks(scales=None), b),
                 (a, blocks(rows=0))):
        assert product(x, y) == B.EINVAL
    for over in (dict(out=None), dict(out=P + 2), dict(type=3), dict(stride=7), dict(mode=4), dict(mode=-1), dict(exact=2), dict(o=order())):
        assert product(a, b, **over) == B.EINVAL
    o, three = order(), blocks(form=B.BLOCKS_SQUARES, count=3)
    for mode, x, y in ((B.PRODUCT_GATHER, a, three), (B.PRODUCT_PLACES, blocks(rows=7), three), (B.PRODUCT_GATHER, blocks(rows=4), sq),
                       (B.PRODUCT_GATHER, blocks(rows=4), b), (B.PRODUCT_OVER, a, b), (B.PRODUCT_OVER, blocks(cols=384), three)):
        assert product(x, y, mode, o=o) == B.EINVAL
    assert product(blocks(rows=4), three, B.PRODUCT_GATHER) == B.EINVAL                  # no order
    raw = blocks(form=B.BLOCKS_RAW, scales=None, stride=200)
    assert product(raw, b) == B.EINVAL                                                   # raw: squares only
    assert product(blocks(form=B.BLOCKS_RAW, rows=17, stride=200), sq) == B.EINVAL
    assert product(blocks(form=B.BLOCKS_RAW, rows=2049, stride=200), three, B.PRODUCT_GATHER, o=order(T=2049)) == B.EINVAL     # 4098 slots
    assert product(blocks(form=B.BLOCKS_RAW, stride=100), sq) == B.EINVAL
    assert product(blocks(rows=0), b) == B.OK


def test_sums_that_are_refused():
    o = order()
    go = lambda y=P, yt=0, n=8, ys=8, w=None, out=P, t=0, s=8: B.lib().asgd_experts_sum(y, yt, n, ys, C.addressof(o), w, out, t, s, None)  # noqa: E731
    for over in (dict(y=None), dict(yt=3), dict(n=0), dict(ys=7), dict(w=P + 2), dict(out=None), dict(t=-1), dict(s=7)):
        assert go(**over) == B.EINVAL
    back = lambda d=P, t=0, s=8, y=P, yt=0, n=8, ys=8, dw=P: B.lib().asgd_experts_sum_backward(d, t, s, y, yt, n, ys, C.addressof(o), dw, None)  # noqa: E731
    for over in (dict(d=None), dict(s=7), dict(y=P + 1), dict(n=0), dict(ys=7), dict(dw=None), dict(dw=P + 2)):
        assert back(**over) == B.EINVAL


def test_tensors_that_are_refused():
    l = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="no CPU fallback"):
        X.route(l, X.Rule(2))
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        X.route(l.double(), X.Rule(2))
    with pytest.raises(ValueError, match="consecutive"):
        X.route(l.t(), X.Rule(2))
    with pytest.raises(ValueError, match="bias"):
        X.route(l, X.Rule(2), bias=torch.zeros(7))
    with pytest.raises(ValueError, match="ids"):
        X.route_backward(l, X.Rule(2), torch.zeros(4, 2), torch.zeros(4, 2))
    with pytest.raises(ValueError, match="ids"):
        X.plan(torch.zeros(4, 2, dtype=torch.int64), 3)
    with pytest.raises(ValueError, match="values"):
        X.Blocks(torch.zeros(4, 100, dtype=torch.uint8), torch.zeros(1, 1), 100)
    with pytest.raises(ValueError, match="scales"):
        X.Blocks(torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(2, 1), 100)
    with pytest.raises(ValueError, match="weights belong"):
        X.quantize(l, weights=torch.zeros(4, 2))
    w = X.Blocks(torch.zeros(2, 4, 128, dtype=torch.uint8), torch.zeros(2, 1, 1), 100)
    with pytest.raises(ValueError, match="one matrix"):
        X.linear(torch.zeros(3, 100), w)
    with pytest.raises(ValueError, match="x:"):
        X.experts(torch.zeros(3, 99), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2), w)
    with pytest.raises(ValueError, match="ids"):
        X.experts(torch.zeros(3, 100), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), w)


def test_the_rules_of_the_tests_hold_by_hand():
    """The 64-bit definitions these tests compare with, on cases worked out by hand."""
    l = torch.tensor([[1.0, 3.0, 3.0, 2.0, -float("inf"), 0.0]])
    assert R.choose(l, "softmax", None, 3, 1, 1, False).tolist() == [[1, 2, 3]]
    assert R.choose(l, "softmax", None, 3, 3, 1, False).tolist() == [[1, 0, -1]]        # groups (1,3) (3,2) (-inf,0): the first 3 wins
    w = R.chosen_weights(l, "sigmoid", None, torch.tensor([[1, 2, -1]]), True, 2.0)
    assert torch.allclose(w, torch.tensor([[1.0, 1.0, 0.0]], dtype=torch.float64))
    q, s = R.to_blocks(torch.tensor([[448.0, 1.0, -17.0]]))
    assert s.tolist() == [[1.0]] and q.float()[0, 0, :3].tolist() == [448.0, 1.0, -16.0]
    assert R.order_of(torch.tensor([[2, 0], [-1, 2]]), 3) == ([0, 1, 1, 3], [0, 1, 1, 2], [1, 0, 3, -1], [1, 0, -1, 2])


def test_direct_experts_that_are_refused():
    x, w = blocks(form=B.BLOCKS_RAW, scales=None, stride=200, type=1), blocks(form=B.BLOCKS_SQUARES, count=3)

    def go(x=x, ids=P, weights=P, k=2, w=w, exact=0, out=P, type=1, stride=8):
        return B.lib().asgd_experts_direct(C.addressof(x), ids, weights, k, C.addressof(w), exact, out, type, stride, None)
    for over in (dict(x=blocks()), dict(x=blocks(form=B.BLOCKS_RAW, rows=17, stride=200)), dict(x=blocks(form=B.BLOCKS_RAW, cols=199, stride=200)), dict(w=blocks()),
                 dict(ids=None), dict(weights=P + 2), dict(k=0), dict(k=65), dict(exact=3), dict(out=None), dict(type=5), dict(stride=7)):
        assert go(**over) == B.EINVAL
