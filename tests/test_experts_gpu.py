"""The products of the experts rows were routed to, on the GPU, against loops over experts in 64 bits."""
import pytest
import torch

from tests import experts_rules as R
from tests.test_experts_blocks_gpu import ROUNDING, TYPES, bounds, data, whole_numbers

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; there is no CPU fallback")
    from paper_1505_04956_amd import experts
    return experts


def routed(T, k, E, seed, skew=False, empty=False):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn(T, E, generator=g) + (torch.randn(E, generator=g) * 2 if skew else 0)
    ids = torch.argsort(l, 1, descending=True)[:, :k].int().contiguous()
    w = torch.rand(T, k, generator=g) + 0.1
    if empty:
        ids[torch.rand(T, k, generator=g) < 0.3] = -1
        ids[T // 2] = -1
    return ids, w


def weights_of(E, N, K, seed):
    return data(E * N, K, seed).view(E, N, K)


CASES = [(1, 1, 1, 1, 1, False), (1, 6, 64, 130, 200, False), (2, 8, 8, 100, 64, False), (5, 3, 7, 65, 300, True), (17, 2, 3, 257, 129, True),
         (130, 4, 9, 140, 260, False), (300, 2, 40, 33, 128, True), (260, 1, 2, 128, 77, False), (64, 5, 100, 20, 40, False)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,E,N,K,empty", CASES)
def test_experts(X, T, k, E, N, K, empty, dtype):
    ids, w = routed(T, k, E, T, skew=True, empty=empty)
    x, mats = data(T, K, 1, dtype), weights_of(E, N, K, 2)
    y = X.experts(x.cuda(), ids.cuda(), w.cuda(), X.quantize_weights(mats.cuda()))
    # and with an order, where few rows would go without
    ways = [y]
    if T <= 16:
        old, X.DIRECT_BYTES = X.DIRECT_BYTES, -1
        ways.append(X.experts(x.cuda(), ids.cuda(), w.cuda(), X.quantize_weights(mats.cuda())))
        X.DIRECT_BYTES = old
    A = R.rounded(x.float())
    want, bound = torch.zeros(T, N, dtype=torch.float64), torch.zeros(T, N, dtype=torch.float64)
    for e in range(E):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if len(t):
            W = R.from_squares(*R.to_squares(mats[e]))[:, :K]
            part, c = A[t] @ W.t(), w[t, j].double()[:, None]
            want.index_add_(0, t, c * part)
            bound.index_add_(0, t, c * (bounds(A[t], W, dtype == torch.float32, torch.float32, part) + (k + 1) * 2 * R.U * part.abs()))
    for y in ways:
        assert y.dtype == dtype and ((y.cpu().double() - want).abs() <= bound * 1.01 + ROUNDING[dtype] * want.abs() + 1e-7).all()
    if empty:
        assert (y[T // 2] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,E,N,K,empty", CASES)
def test_gradients_are_the_formulas(X, T, k, E, N, K, empty, dtype):
    ids, w = routed(T, k, E, T + 1, skew=True, empty=empty)
    x, d, mats = data(T, K, 1, dtype), data(T, N, 5, dtype), weights_of(E, N, K, 2)
    _, kept = X.experts(x.cuda(), ids.cuda(), w.cuda(), X.quantize_weights(mats.cuda()), train=True)
    d_x, d_w, d_weights = X.experts_backward(d.cuda(), kept, X.quantize_weights(mats.cuda(), turned=True))
    A, D = R.rounded(x.float()), d.double()
    f64 = torch.float64
    wx, bx = torch.zeros(T, K, dtype=f64), torch.zeros(T, K, dtype=f64)
    ww, bw = torch.zeros(T, k, dtype=f64), torch.zeros(T, k, dtype=f64)
    for e in range(E):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if not len(t):
            assert (d_w[e] == 0).all()
            continue
        W = R.from_squares(*R.to_squares(mats[e]))[:, :K]
        part = A[t] @ W.t()
        ww[t, j] = (D[t] * part).sum(1)
        bw[t, j] = (D[t].abs() * bounds(A[t], W, True, torch.float32, part)).sum(1) + (N / 64 + 10) * 2 * R.U * (D[t] * part).abs().sum(1)
        rows = w[t, j][:, None] * d[t].float()
        Q = R.rounded(rows)
        back = Q @ W
        wx.index_add_(0, t, back)
        bx.index_add_(0, t, bounds(Q, W.t().contiguous(), dtype == torch.float32, torch.float32, back) + (k + 1) * 2 * R.U * back.abs())
        # blocks of 128 of the expert's own rows, in the order of slots
        Dt, Xt = R.rounded(rows.t()), R.rounded(x[t].float().t())
        want = Dt @ Xt.t()
        assert ((d_w[e].cpu().double() - want).abs() <= bounds(Dt, Xt, True, torch.float32, want)).all()
    assert ((d_x.cpu().double() - wx).abs() <= bx * 1.01 + ROUNDING[dtype] * wx.abs() + 1e-7).all()
    assert ((d_weights.cpu().double() - ww).abs() <= bw * 1.01 + 1e-30).all()
    assert (d_weights.cpu()[ids < 0] == 0).all()


def test_gradients_are_those_of_differences(X):
    """Where 8 bits hold everything the experts are linear in x, in w and in the weights: steps of one differ by the gradient."""
    T, k, E, N, K = 140, 2, 3, 130, 140
    ids, _ = routed(T, k, E, 7)
    weights = torch.ones(T, k)
    x, mats, d = whole_numbers(T, K, 1), whole_numbers(E * N, K, 2).view(E, N, K).clone(), whole_numbers(T, N, 3)
    mats[:, 0], mats[:, 128] = 448.0, 448.0
    x[:, :] = whole_numbers(T, K, 1)
    # every expert's blocks of rows need a 448 of their own: the columns' first rows in the expert's order
    for e in range(E):
        t, _ = torch.nonzero(ids == e, as_tuple=True)
        x[t[::128]], d[t[::128]] = 448.0, 448.0
    run = lambda x, m, c: X.experts(x.cuda(), ids.cuda(), c.cuda(), X.quantize_weights(m.cuda()))  # noqa: E731
    f = lambda x, m, c: (run(x, m, c).double() * d.cuda().double()).sum().item()  # noqa: E731
    _, kept = X.experts(x.cuda(), ids.cuda(), weights.cuda(), X.quantize_weights(mats.cuda()), train=True)
    d_x, d_w, d_weights = X.experts_backward(d.cuda(), kept, X.quantize_weights(mats.cuda(), turned=True))
    plain = [t for t in range(T) if x[t, 1] != 448.0]
    for t, j in ((plain[0], 1), (plain[40], 139), (plain[-1], 70)):
        up, down = x.clone(), x.clone()
        up[t, j] += 1
        down[t, j] -= 1
        assert (f(up, mats, weights) - f(down, mats, weights)) / 2 == d_x[t, j].item()
    for e, n, j in ((0, 1, 1), (1, 129, 139), (2, 64, 30)):
        up, down = mats.clone(), mats.clone()
        up[e, n, j] += 1
        down[e, n, j] -= 1
        assert (f(x, up, weights) - f(x, down, weights)) / 2 == d_w[e, n, j].item()
    for t, j in ((0, 0), (77, 1), (139, 0)):
        up, down = weights.clone(), weights.clone()
        up[t, j] += 1
        down[t, j] -= 1
        # (sums of numbers beyond 2^24: equal to the roundings of N products and of their sum)
        size = (kept.y[kept.plan.places.view(T, k)[t, j]].double() * d[t].cuda().double()).abs().sum().item()
        assert abs((f(x, mats, up) - f(x, mats, down)) / 2 - d_weights[t, j].item()) <= (N / 64 + 10) * 2 * R.U * size


@pytest.mark.parametrize("dtype", TYPES)
def test_sum_of_strided_rows(X, dtype):
    ids, w = routed(20, 3, 6, 2, empty=True)
    p = X.plan(ids.cuda(), 6)
    y = data(60, 300, 3, dtype).cuda()[:, 7:240]
    got = X.experts_sum(y, p, torch.float32, weights=w.cuda()).cpu().double()
    places = p.places.cpu().view(20, 3).long()
    rows = y.cpu().double()[places.clamp_min(0)] * (places >= 0)[:, :, None]
    want = (rows * w.double()[:, :, None]).sum(1)
    assert ((got - want).abs() <= 8 * R.U * (rows.abs() * w.double()[:, :, None]).sum(1)).all()
    d = data(20, 300, 4, dtype).cuda()[:, 3:236]
    got = X.experts_sum_backward(d, y, p).cpu().double()
    want = (rows * d.cpu().double()[:, None]).sum(2)
    assert ((got - want).abs() <= (233 / 64 + 12) * 2 * R.U * (rows * d.cpu().double()[:, None]).abs().sum(2)).all()


def test_places_that_are_not_in_use_hold_anything(X):
    """What memory held before must not reach a result: slots without experts, rows of no place."""
    T, k, E, N, K = 40, 4, 5, 100, 130
    ids, w = routed(T, k, E, 3, empty=True)
    x, d, mats = data(T, K, 1), data(T, N, 2), weights_of(E, N, K, 3)
    wq, wt = X.quantize_weights(mats.cuda()), X.quantize_weights(mats.cuda(), turned=True)

    def all_of_it():
        y, kept = X.experts(x.cuda(), ids.cuda(), w.cuda(), wq, train=True)
        return (y, *X.experts_backward(d.cuda(), kept, wt))
    first = [t.clone() for t in all_of_it()]
    junk = [torch.full((n,), float("nan"), device="cuda") for n in (1 << 12, 1 << 14, 1 << 16, 1 << 18, 1 << 20)]
    junk += [torch.full((n,), float("nan"), device="cuda") for n in (T * k * N, T * k * K, E * N * K)]
    del junk
    for a, b in zip(first, all_of_it()):
        assert torch.isfinite(b).all() and torch.equal(a, b)


def test_no_tokens(X):
    mats = weights_of(3, 40, 50, 1)
    x, ids, w = torch.empty(0, 50, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, device="cuda")
    y, kept = X.experts(x, ids, w, X.quantize_weights(mats.cuda()), train=True)
    d_x, d_w, d_weights = X.experts_backward(torch.empty(0, 40, device="cuda"), kept, X.quantize_weights(mats.cuda(), turned=True))
    assert y.shape == (0, 40) and d_x.shape == (0, 50) and d_weights.shape == (0, 2) and (d_w == 0).all() and d_w.shape == (3, 40, 50)


def test_in_a_graph_with_other_routes(X):
    """One capture serves whatever the router says: nothing of the order is known to the host."""
    T, k, E, N, K = 50, 3, 8, 130, 256
    wq = X.quantize_weights(weights_of(E, N, K, 3).cuda())
    x = data(T, K, 1).cuda()
    ids, w = (t.cuda() for t in routed(T, k, E, 1))
    X.experts(x, ids, w, wq)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = X.experts(x, ids, w, wq)
    for seed in (2, 3, 4):
        i, c = routed(T, k, E, seed, skew=True, empty=seed == 3)
        ids.copy_(i)
        w.copy_(c)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, X.experts(x.clone(), i.cuda(), c.cuda(), wq))


def test_a_clustering_becomes_a_routed_model(X):
    """Centroids by ASGD, then routing, experts and both gradients in a training loop: better than any single linear map."""
    from paper_1505_04956_amd import clusterwise
    losses, single = clusterwise.run(samples=60_000, steps=60, batch=4096)
    assert losses[-1] < 0.75 * losses[0] and sum(losses[-5:]) / 5 < single


def test_gathered_rows_more_than_32_bits_apart(X):
    """Rows of one tile that lie at both ends of more than 2^32 bytes of 8-bit rows."""
    T, K, N, E = 280_000, 16_384, 24, 3
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB")
    x = torch.zeros((T, K), dtype=torch.bfloat16, device="cuda")
    at = [0, 1, 140_000, 279_998, 279_999]
    x[at] = data(5, K, 8).to(torch.bfloat16).cuda()
    ids = torch.zeros((T, 1), dtype=torch.int32, device="cuda")
    ids[2:140_000] = 1
    ids[140_001:279_998] = 1                          # expert 0: a few rows at the ends; expert 2: none
    w, weights = X.quantize_weights(weights_of(E, N, K, 2).cuda()), torch.ones((T, 1), device="cuda")
    y = X.experts(x, ids, weights, w)
    few = [0, 1, 140_000, 279_998, 279_999] + list(range(2, 400))
    part = X.experts(x[few], ids[few], weights[few], w)
    assert torch.equal(y[at], part[:5]) and int((y.float().abs().sum(1) > 0).sum()) == 5
