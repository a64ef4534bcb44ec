"""What the calls of 4-bit blocks, layers of experts and gradients refuse.  No GPU is needed: nothing that is refused is enqueued."""
import ctypes as C
from array import array

import pytest
import torch

from paper_1505_04956_amd import binding as B
from paper_1505_04956_amd import experts as X
from paper_1505_04956_amd import gradients as G
from paper_1505_04956_amd import layer as L
from paper_1505_04956_amd import micro as M
from tests import micro_rules as Q

P = 1 << 20                                                         # an address that is never used


def blocks(rows=8, cols=300, form=B.BLOCKS_FOURS, count=1, values=P, scales=P, type=0, stride=0):
    return B.asgd_blocks(values, scales, rows, cols, form, count, type, stride)


def order(T=8, k=2, E=3):
    return B.asgd_route_order(T, k, E, P, P, P, P)


def raw(rows=8, cols=300, **over):
    return blocks(rows, cols, B.BLOCKS_RAW, scales=None, **{"type": 1, "stride": cols, **over})


def test_bringing_to_four_bits_that_is_refused():
    def go(out, x=P, type=1, rows=8, cols=300, stride=300, turned=0, o=None, weights=None):
        return B.lib().asgd_block_quantize(x, type, rows, cols, stride, turned, None if o is None else C.addressof(o), weights, C.addressof(out), None)
    for out in (blocks(values=None), blocks(scales=None), blocks(values=P + 8), blocks(scales=P + 4), blocks(rows=9), blocks(cols=299), blocks(form=3), blocks(form=5), blocks(count=0),
                blocks(count=1025)):
        assert go(out) == B.EINVAL
    for over in (dict(x=None), dict(x=P + 1), dict(type=4), dict(rows=-1), dict(cols=0), dict(stride=299), dict(turned=1), dict(turned=2), dict(weights=P), dict(o=order())):
        assert go(blocks(), **over) == B.EINVAL
    assert go(blocks(rows=0), rows=0) == B.OK
    big = (1 << 30) // 8 + 1
    assert go(blocks(rows=big, count=8), rows=big) == B.EINVAL


def test_giving_back_that_is_refused():
    def go(x, out=P, type=0, stride=300):
        return B.lib().asgd_block_expand(C.addressof(x), out, type, stride, None)
    for x in (blocks(form=B.BLOCKS_SQUARES), blocks(form=B.BLOCKS_ROWS), raw(), blocks(values=None), blocks(scales=P + 4), blocks(rows=-1)):
        assert go(x) == B.EINVAL
    for over in (dict(out=None), dict(out=P + 2), dict(type=3), dict(stride=299)):
        assert go(blocks(), **over) == B.EINVAL
    assert go(blocks(rows=0)) == B.OK


def test_products_that_are_refused():
    def go(a, b, mode=B.PRODUCT_ALL, o=None, exact=0, out=P, type=0, stride=8):
        return B.lib().asgd_block_product(C.addressof(a), C.addressof(b), mode, exact, None if o is None else C.addressof(o), out, type, stride, None)
    squares, rows = blocks(form=B.BLOCKS_SQUARES), blocks(form=B.BLOCKS_ROWS)
    for a, b in ((blocks(), squares), (blocks(), rows), (rows, blocks()), (squares, blocks()), (blocks(cols=301), blocks()), (blocks(count=2), blocks()), (blocks(), blocks(count=2)),
                 (blocks(), raw()), (raw(rows=17), blocks()), (blocks(), blocks(rows=0))):
        assert go(a, b) == B.EINVAL
        assert B.asgd_block_product_form(a, b, B.PRODUCT_ALL, 0, None) == B.PRODUCT_FORM_NONE
    for over in (dict(out=None), dict(out=P + 1), dict(type=3), dict(stride=7), dict(exact=2), dict(o=order()), dict(mode=B.PRODUCT_OVER), dict(mode=7), dict(mode=B.PRODUCT_GATHER)):
        assert go(blocks(), blocks(), **over) == B.EINVAL
    o, w = order(), blocks(count=3)
    for a, b, mode in ((blocks(rows=9), w, B.PRODUCT_GATHER), (blocks(rows=8), w, B.PRODUCT_PLACES), (blocks(rows=16, count=3), w, B.PRODUCT_PLACES), (blocks(), blocks(count=2), B.PRODUCT_GATHER),
                       (raw(rows=16), w, B.PRODUCT_PLACES), (blocks(rows=64, cols=512), blocks(rows=64, cols=512), B.PRODUCT_OVER)):
        assert go(a, b, mode, o) == B.EINVAL
    # which kernel
    form = lambda rows, outs, cols: B.asgd_block_product_form(blocks(rows, cols), blocks(outs, cols), B.PRODUCT_ALL, 0, None)  # noqa: E731
    assert form(32, 4096, 4096) == B.PRODUCT_FORM_FEW and form(33, 100, 100) not in (B.PRODUCT_FORM_FEW, B.PRODUCT_FORM_NONE)
    assert form(8192, 8192, 8192) == B.PRODUCT_FORM_TILES_256
    assert B.asgd_block_product_form(raw(), blocks(), B.PRODUCT_ALL, 0, None) == B.PRODUCT_FORM_FEW


def test_experts_of_few_rows_that_are_refused():
    def go(x, w, ids=P, weights=P, k=2, out=P, stride=8):
        return B.lib().asgd_experts_direct(C.addressof(x), ids, weights, k, C.addressof(w), 1, out, 0, stride, None)
    w = blocks(count=3)
    for x, m in ((raw(rows=4097), w), (raw(rows=17), blocks(form=B.BLOCKS_SQUARES, count=3)), (raw(cols=299), w), (blocks(), w), (raw(), blocks(form=B.BLOCKS_ROWS))):
        assert go(x, m) == B.EINVAL
    for over in (dict(ids=None), dict(weights=None), dict(ids=P + 2), dict(k=0), dict(k=65), dict(out=None), dict(stride=7)):
        assert go(raw(), w, **over) == B.EINVAL
    assert go(raw(rows=0), w) == B.OK


@pytest.mark.parametrize("form", [B.BLOCKS_FOURS, B.BLOCKS_SQUARES])
def test_layers_that_are_refused(form):
    T, E, D, H, N, k = 8, 6, 300, 50, 70, 2
    up, down = blocks(2 * H, D, form, E), blocks(N, H, form, E)
    other = B.BLOCKS_SQUARES if form == B.BLOCKS_FOURS else B.BLOCKS_FOURS

    def go(x=None, up=up, down=down, rule=None, logits=P, ltype=0, lstride=E, bias=None, act=0, ids=P, weights=P, out=P, type=1, stride=N, work=P, size=None):
        x, rule = x or raw(T, D), rule or B.asgd_route_rule(k, 0, 1, 1, 0, 1, 1.0)
        size = B.asgd_experts_layer_bytes(T, k, E, D, H) if size is None else size
        return B.lib().asgd_experts_layer(C.addressof(x), logits, ltype, lstride, bias, C.addressof(rule), C.addressof(up), C.addressof(down), act, ids, weights, out, type, stride,
                                          work, size, None)
    need = B.asgd_experts_layer_bytes(T, k, E, D, H)
    assert need >= T * k * H * 4
    for over in (dict(x=raw(17, D)), dict(x=raw(T, D + 1)), dict(x=blocks(T, D)), dict(up=blocks(2 * H + 1, D, form, E)), dict(up=blocks(2 * H, D, form, E + 1)), dict(up=blocks(2 * H, D, other, E)),
                 dict(down=blocks(N, H + 1, form, E)), dict(down=blocks(0, H, form, E)), dict(up=blocks(2 * H, D, B.BLOCKS_ROWS), down=blocks(N, H, B.BLOCKS_ROWS)),
                 dict(rule=B.asgd_route_rule(E + 1, 0, 1, 1, 0, 1, 1.0)), dict(rule=B.asgd_route_rule(0, 0, 1, 1, 0, 1, 1.0)), dict(rule=B.asgd_route_rule(k, 2, 1, 1, 0, 1, 1.0)),
                 dict(logits=None), dict(logits=P + 2), dict(ltype=3), dict(lstride=E - 1), dict(bias=P + 2), dict(act=2), dict(act=-1), dict(ids=None), dict(ids=P + 2), dict(weights=None),
                 dict(weights=P + 1), dict(out=None), dict(out=P + 1), dict(type=3), dict(stride=N - 1), dict(work=None), dict(work=P + 8), dict(size=need - 1)):
        assert go(**over) == B.EINVAL, over
    assert go(x=raw(0, D)) == B.OK
    for sizes in ((17, 2, 5, 9, 9), (1, 0, 5, 9, 9), (1, 65, 5, 9, 9), (1, 1, 0, 9, 9), (1, 1, 1025, 9, 9), (1, 1, 5, 0, 9), (1, 1, 5, 9, 0), (-1, 1, 5, 9, 9)):
        assert B.asgd_experts_layer_bytes(*sizes) == 0


def spans(*runs):
    return array("q", [v for r in runs for v in r])


def test_gradients_that_are_refused():
    lib = B.lib()

    def go(runs, out=None, limit=1.0, norm=P, work=P, size=1 << 30, count=None):
        n = len(runs) // 3 if count is None else count
        return lib.asgd_gradient_clip(runs.buffer_info()[0], None if out is None else out.buffer_info()[0], n, limit, norm, work, size, None)
    A = 1 << 24
    good = spans((A, 100, 0), (A + 400, 10, 1))
    assert B.asgd_gradient_bytes(2) > 0 and B.asgd_gradient_bytes(-1) == B.asgd_gradient_bytes((1 << 20) + 1) == 0
    for bad in (spans((A, -1, 0)), spans((A, 5, 3)), spans((A, 5, -1)), spans((A + 2, 5, 0)), spans((A + 1, 5, 1)), spans((0, 5, 0)), spans((A, 1 << 41, 1))):
        assert go(bad) == B.EINVAL
        assert lib.asgd_gradient_norm(bad.buffer_info()[0], 1, P, P, 1 << 30, None) == B.EINVAL
    for over in (dict(limit=-1.0), dict(limit=float("nan")), dict(norm=None), dict(norm=P + 2), dict(work=None), dict(work=P + 8), dict(size=8), dict(count=-1), dict(count=(1 << 20) + 1)):
        assert go(good, **over) == B.EINVAL, over
    for out in (spans((A, 100, 0), (A + 404, 10, 1)), spans((A, 99, 0), (A + 400, 10, 1)), spans((A, 100, 1), (A + 400, 10, 1)), spans((A + (1 << 20), 100, 0), (A + (1 << 20) + 396, 10, 1)),
                spans((A + 400, 100, 0), (A + (1 << 20), 10, 1))):
        assert go(good, out) == B.EINVAL
    assert go(spans((A, 100, 0), (A + 398, 10, 1))) == B.EINVAL and go(spans((A, 100, 0), (A, 100, 0))) == B.EINVAL


def fours(*shape, cols):
    return M.Micro(torch.zeros(*shape, 128 * -(-cols // 256), dtype=torch.uint8), torch.zeros(*shape, 8 * -(-cols // 256), dtype=torch.uint8), cols)


def test_tensors_that_are_refused():
    for values, scales, cols in ((torch.zeros(4, 128), torch.zeros(4, 8, dtype=torch.uint8), 200), (torch.zeros(4, 128, dtype=torch.int8), torch.zeros(4, 8, dtype=torch.uint8), 200),
                                 (torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 8), 200), (torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 8, dtype=torch.uint8), 300),
                                 (torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(5, 8, dtype=torch.uint8), 200), (torch.zeros(128, dtype=torch.uint8), torch.zeros(8, dtype=torch.uint8), 200),
                                 (torch.zeros(8, 128, dtype=torch.uint8)[::2], torch.zeros(4, 8, dtype=torch.uint8), 200)):
        with pytest.raises(ValueError, match="values|scales"):
            M.Micro(values, scales, cols)
    w, many = fours(6, cols=200), fours(3, 6, cols=200)
    assert (w.rows, w.cols, w.count, many.rows, many.count) == (6, 200, 1, 6, 3)
    for name in ("values", "scales", "rows", "cols", "count"):
        with pytest.raises(AttributeError):
            setattr(w, name, getattr(w, name))
    x, ids, c = torch.zeros(4, 200), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    squares = X.Blocks(torch.zeros(3, 6, 256, dtype=torch.uint8), torch.zeros(3, 1, 2), 200)
    for call in (lambda: M.linear(x[:, :199], w), lambda: M.linear(x, many), lambda: M.linear(x, squares), lambda: M.linear(x[0], w), lambda: M.experts(x, ids[:3], c, many),
                 lambda: M.experts(x, ids, c[:3], many), lambda: M.experts(x, ids.long(), c, many), lambda: M.experts(x, ids, c.double(), many), lambda: M.experts(x, ids, c, squares),
                 lambda: M.quantize(torch.zeros(3, 4, 6).transpose(1, 2)), lambda: M.quantize(torch.zeros(6, 4).t()), lambda: M.quantize(torch.zeros(4, 6, dtype=torch.float64)),
                 lambda: M.quantize(torch.zeros(4)), lambda: M.expand(w, torch.float64)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: M.linear(x, w), lambda: M.experts(x, ids, c, many), lambda: M.quantize(x), lambda: M.expand(w), lambda: M.product(w, w, torch.float32)):
        with pytest.raises(ValueError, match="no CPU fallback"):
            call()


def test_layers_of_tensors_that_are_refused():
    E, D, H, N = 3, 200, 40, 30
    up, down, rule = fours(E, 2 * H, cols=D), fours(E, N, cols=H), X.Rule(2)
    up8 = X.Blocks(torch.zeros(E, 2 * H, 256, dtype=torch.uint8), torch.zeros(E, 1, 2), D)
    x, l = torch.zeros(4, D), torch.zeros(4, E)
    for call in (lambda: L.layer(x, l, rule, up8, down), lambda: L.layer(x, l, rule, up, up), lambda: L.layer(x, l, rule, down, up), lambda: L.layer(x[:, :100], l, rule, up, down),
                 lambda: L.layer(torch.zeros(17, D), torch.zeros(17, E), rule, up, down), lambda: L.layer(x, l[:3], rule, up, down), lambda: L.layer(x, l[:, :2], rule, up, down),
                 lambda: L.layer(x, l.double(), rule, up, down), lambda: L.layer(x, l, rule, up, down, bias=torch.zeros(E + 1)), lambda: L.layer(x, l, rule, up._c, down),
                 lambda: L.layer(x.t(), l, rule, up, down)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError, match="no CPU fallback"):
        L.layer(x, l, rule, up, down)
    for call in (lambda: L.layer(x.clone().requires_grad_(True), l, rule, up, down), lambda: L.layer(x, l.clone().requires_grad_(True), rule, up, down),
                 lambda: L.layer(x, l, rule, up, down, bias=torch.zeros(E, requires_grad=True)), lambda: M.linear(x.clone().requires_grad_(True), fours(6, cols=D)),
                 lambda: M.quantize(x.clone().requires_grad_(True)), lambda: M.quantize(torch.zeros(2, 3, 4, requires_grad=True)),
                 lambda: G.norm([x.clone().requires_grad_(True)]), lambda: G.clip([x], 1.0, out=[x.clone().requires_grad_(True)])):
        with pytest.raises(ValueError, match="gradient"):
            call()


def test_gradients_of_tensors_that_are_refused():
    x = torch.zeros(4, 6)
    for call in (lambda: G.norm([]), lambda: G.norm([x.t()]), lambda: G.norm([x.double()]), lambda: G.norm([x[:, :3]]), lambda: G.clip([x], -1.0), lambda: G.clip([x], float("nan")),
                 lambda: G.clip([x], 1.0, out=[]), lambda: G.clip([x], 1.0, out=[x[:3]]), lambda: G.clip([x], 1.0, out=[x.t()]), lambda: G.clip([x], 1.0, out=[x, x])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError, match="no CPU fallback"):
        G.norm([x])


def test_the_definition_of_four_bits():
    """The oracle's own steps at numbers that are worked out by hand."""
    x = torch.zeros(5, 32)
    x[0, :4] = torch.tensor([6.0, 0.25, 0.75, -2.5])                # scale 1
    x[1, :2] = torch.tensor([6.99, 5.0])                            # scale 1, cut
    x[2, :3] = torch.tensor([7.0, 1.0, 0.5])                        # scale 2
    x[3, 0] = 1.0                                                   # scale 1 / 4: 4
    code, s = Q.to_four(x)
    assert s[:, 0].tolist() == [127, 127, 128, 125, 1] and s[0, 1] == 1
    assert code[0, :4].tolist() == [7, 0, 2, 12] and code[1, :2].tolist() == [7, 6] and code[2, :3].tolist() == [6, 1, 0] and code[3, 0] == 6
    assert Q.four(x)[2, :3].tolist() == [8.0, 1.0, 0.0]


def test_what_clipping_writes_counts_as_written(monkeypatch):
    """The library writes through addresses, so clip() moves the versions of the tensors that it writes, of no others, and of none where it refuses.  (The
    library and the stream stand aside here: nothing is computed.)"""
    calls = []
    monkeypatch.setattr(X, "_stream", lambda t: 0)
    monkeypatch.setattr(B, "asgd_gradient_clip", lambda *a: calls.append(a))
    monkeypatch.setattr(B, "asgd_gradient_norm", lambda *a: calls.append(a))
    versions = lambda tensors: [t._version for t in tensors]  # noqa: E731
    grads, out = [torch.zeros(4), torch.zeros(3, 2, dtype=torch.bfloat16), torch.zeros(0)], [torch.zeros(4), torch.zeros(6), torch.zeros(0)]
    G.norm(grads)
    assert versions(grads) == [0, 0, 0]
    G.clip(iter(grads), 1.0)
    assert all(v > 0 for v in versions(grads)) and versions(out) == [0, 0, 0]
    was = versions(grads)
    G.clip(grads, 1.0, out=iter(out))
    assert versions(grads) == was and all(v > 0 for v in versions(out))
    G.clip(grads, 1.0, out=[grads[0], out[1], out[2]])
    assert grads[0]._version > was[0] and versions(grads[1:]) == was[1:]
    # a view's is its base's, and a leaf's moves where no gradients are recorded
    base, leaf = torch.zeros(10), torch.zeros(4, requires_grad=True)
    with torch.no_grad():
        G.clip([base[2:5], leaf], 1.0)
    assert base._version > 0 and leaf._version > 0
    # tensors of inference mode have none
    with torch.inference_mode():
        free = torch.zeros(4)
        G.clip([free, base], 1.0)
    G.clip([free], 1.0)
    # what was saved and is clipped before its backward
    a, b = torch.ones(4, requires_grad=True), torch.ones(4)
    y = (a * b).sum()
    G.clip([b], 1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    assert len(calls) == 8

    def refused(*a):
        raise B.AsgdError(B.EINVAL, "asgd_gradient_clip")
    monkeypatch.setattr(B, "asgd_gradient_clip", refused)
    was = versions(grads + out)
    with pytest.raises(B.AsgdError):
        G.clip(grads, 1.0, out=out)
    assert versions(grads + out) == was


def test_what_is_written_shares_memory_with_nothing():
    """Wherever it lies among runs that are only read, inside long ones and behind short ones that lie in them too."""
    A, F = 1 << 24, 1 << 25
    go = lambda runs, out: B.lib().asgd_gradient_clip(runs.buffer_info()[0], out.buffer_info()[0], len(runs) // 3, 1.0, P, P, 1 << 30, None)  # noqa: E731
    for runs, out in ((spans((A, 1000, 0), (A + 40, 10, 0)), spans((F, 1000, 0), (A + 2000, 10, 0))), (spans((A + 40, 10, 0), (A, 1000, 0)), spans((A + 3996, 10, 0), (F, 1000, 0))),
                      (spans((A, 100, 0), (A, 100, 0)), spans((A, 100, 0), (F, 100, 0))), (spans((A, 100, 0), (A, 100, 0)), spans((F, 100, 0), (F, 100, 0))),
                      (spans((A, 100, 0), (A, 100, 0)), spans((A, 100, 0), (A, 100, 0))), (spans((A + 100, 50, 0), (A, 1000, 0)), spans((A + 100, 50, 0), (F, 1000, 0))),
                      (spans((A + 4, 10, 0), (A + 8, 10, 0), (F, 2, 0)), spans((F + 8, 10, 0), (F + 400, 10, 0), (A, 2, 0))),
                      (spans((F, 1000, 0), (A, 2, 0)), spans((A, 1000, 0), (A + 500, 2, 0)))):
        assert out[1::3] == runs[1::3]
        assert go(runs, out) == B.EINVAL
