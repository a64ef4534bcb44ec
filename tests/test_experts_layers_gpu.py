"""Experts of two products with an activation between them, from the pieces: what unused places hold must not reach a result, and each
step is that of its formula in 64 bits."""
import pytest
import torch

from tests import experts_rules as R
from tests.test_experts_blocks_gpu import bounds, data
from tests.test_experts_gpu import routed, weights_of

pytestmark = pytest.mark.gpu
F32 = torch.float32


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; there is no CPU fallback")
    from paper_1505_04956_amd import experts
    return experts


def forward(X, x, order, weights, up, down):
    """(out, pre, h): pre = up x and h = pre sigmoid(pre) at places, out the weighted sum of down h."""
    pre = X.product(X.quantize(x), up, F32, order, gather=True)
    h = pre * torch.sigmoid(pre)
    return X.experts_sum(X.product(X.quantize(h), down, F32, order), order, F32, weights), pre, h


def backward(X, x, d, order, by_slot, weights, pre, h, up_turned, down_turned):
    """Gradients of up, down and x; what is at places goes to slots (an order of one choice a row) to be turned."""
    rows, turned = X.quantize(d, plan=order, weights=weights), X.quantize(d, turned=True, plan=order, weights=weights)
    d_down = X.product_over(turned, X.quantize(X.experts_sum(h, by_slot, F32), turned=True, plan=by_slot), order)
    d_h = X.product(rows, down_turned, F32, order)
    s = torch.sigmoid(pre)
    d_pre = d_h * (s + pre * s * (1 - s))
    slots = X.experts_sum(d_pre, by_slot, F32)
    d_up = X.product_over(X.quantize(slots, turned=True, plan=by_slot), X.quantize(x, turned=True, plan=order), order)
    return d_up, d_down, X.experts_sum(X.product(X.quantize(d_pre), up_turned, F32, order), order, F32), d_pre


@pytest.mark.parametrize("T,k,E,K,H,N", [(1, 2, 4, 64, 128, 64), (70, 3, 9, 130, 200, 100), (900, 2, 4, 260, 300, 130)])
def test_two_products_and_an_activation(X, T, k, E, K, H, N):
    ids, weights = routed(T, k, E, T, skew=True, empty=T > 1)
    x, d = data(T, K, 1), data(T, N, 2)
    up, down = weights_of(E, H, K, 3) / 16, weights_of(E, N, H, 4) / 16
    order, by_slot, w = X.plan(ids.cuda(), E), X.plan(ids.reshape(-1, 1).cuda(), E), weights.cuda()
    assert torch.equal(order.slots, by_slot.slots) and torch.equal(order.blocks, by_slot.blocks)
    q = [X.quantize_weights(m.cuda(), turned=t) for m in (up, down) for t in (False, True)]

    def all_of_it():
        out, pre, h = forward(X, x.cuda(), order, w, q[0], q[2])
        return (out, pre, h, *backward(X, x.cuda(), d.cuda(), order, by_slot, w, pre, h, q[1], q[3]))
    first = [t.clone() for t in all_of_it()]
    for n in (T * k * K, T * k * H, T * k * N, T * N, T * K, E * H * K, E * N * H):
        for _ in range(6):
            torch.full((n,), float("nan"), device="cuda")
    again = all_of_it()
    used = order.slots >= 0
    for i, (a, b) in enumerate(zip(first, again)):
        a, b = (a[used], b[used]) if i in (1, 2, 6) else (a, b)                # (at places)
        assert torch.isfinite(b).all() and torch.equal(a, b)
    out, pre, h, d_up, d_down, d_x, d_pre = (t.cpu() for t in again)

    places = order.places.cpu().view(T, k)
    A, zero = R.rounded(x), torch.zeros
    want, off = zero(T, N, dtype=torch.float64), zero(T, N, dtype=torch.float64)
    want_x, off_x = zero(T, K, dtype=torch.float64), zero(T, K, dtype=torch.float64)
    for e in range(E):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if not len(t):
            assert (d_up[e] == 0).all() and (d_down[e] == 0).all()
            continue
        U, D = R.from_squares(*R.to_squares(up[e]))[:, :K], R.from_squares(*R.to_squares(down[e]))[:, :H]
        at, c = places[t, j].long(), weights[t, j].double()[:, None]
        part = A[t] @ U.t()
        assert ((pre[at].double() - part).abs() <= bounds(A[t], U, True, F32, part)).all()
        Hq = R.rounded(h[at])                                                 # (the step after takes what this one gave)
        part = Hq @ D.t()
        want.index_add_(0, t, c * part)
        off.index_add_(0, t, c * (bounds(Hq, D, True, F32, part) + (k + 1) * 2 * R.U * part.abs()))
        rows = weights[t, j][:, None] * d[t]
        Rt, Ht = R.rounded(rows.t()), R.rounded(h[at].t())
        part = Rt @ Ht.t()
        assert ((d_down[e].double() - part).abs() <= bounds(Rt, Ht, True, F32, part)).all()
        Pt, Xt = R.rounded(d_pre[at].t()), R.rounded(x[t].t())
        part = Pt @ Xt.t()
        assert ((d_up[e].double() - part).abs() <= bounds(Pt, Xt, True, F32, part)).all()
        P = R.rounded(d_pre[at])
        part = P @ U
        want_x.index_add_(0, t, part)
        off_x.index_add_(0, t, bounds(P, U.t().contiguous(), True, F32, part) + (k + 1) * 2 * R.U * part.abs())
    assert ((out.double() - want).abs() <= 1.01 * off + 1e-30).all()
    assert ((d_x.double() - want_x).abs() <= 1.01 * off_x + 1e-30).all()


@pytest.mark.parametrize("T,k,E", [(1, 2, 8), (300, 2, 8), (1000, 6, 64)])
def test_from_logits_to_gradients(X, T, k, E):
    """Routing and experts together, rows that are padded among them: ids and weights go from one to the other as they are."""
    K, N = 200, 150
    g = torch.Generator().manual_seed(T)
    l, x, d = torch.randn(T, E, generator=g), data(T, K, 1), data(T, N, 2)
    if T > 1:
        l[::7], x[::7], d[::7] = -float("inf"), float("nan"), float("inf")     # (padding, whatever it holds)
    mats, rule = weights_of(E, N, K, 3), X.Rule(k, scale=1.5)
    ids, w = X.route(l.cuda(), rule)
    y, kept = X.experts(x.cuda(), ids, w, X.quantize_weights(mats.cuda()), train=True)
    d_x, d_w, d_weights = X.experts_backward(d.cuda(), kept, X.quantize_weights(mats.cuda(), turned=True))
    d_l = X.route_backward(l.cuda(), rule, ids, d_weights)
    for t in (y, d_x, d_w, d_weights, d_l):
        assert torch.isfinite(t).all()
    real = ~torch.isinf(l).all(1)
    for t in (y, d_x, d_weights, d_l):
        assert (t[(~real).cuda()] == 0).all()
    some = [t.cuda() for t in (l[real], x[real], d[real])]
    ids, w = X.route(some[0], rule)
    y2, kept = X.experts(some[1], ids, w, X.quantize_weights(mats.cuda()), train=True)
    back = X.experts_backward(some[2], kept, X.quantize_weights(mats.cuda(), turned=True))
    assert torch.equal(y[real.cuda()], y2) and torch.equal(d_x[real.cuda()], back[0]) and torch.equal(d_w, back[1]) and torch.equal(d_weights[real.cuda()], back[2])


def test_a_clustering_with_a_map_for_all(X):
    """The example with --shared: routing, experts and a layer that every row passes through, each with its gradient, in one training loop."""
    from paper_1505_04956_amd import clusterwise
    losses, single = clusterwise.run(samples=60_000, steps=60, batch=4096, shared=True)
    assert losses[-1] < 0.75 * losses[0] and sum(losses[-5:]) / 5 < single
