"""How the products of a block are summed: what callers get without asking, what they can ask for, what the 8-bit instruction drops."""
import pytest
import torch

from tests import experts_rules as R
from tests.test_experts_blocks_gpu import ROUNDING, TYPES, bounds, data
from tests.test_experts_gpu import routed, weights_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; there is no CPU fallback")
    from paper_1505_04956_amd import experts
    return experts


def cancelling(rows, cols):
    """(x, w): in every eight neighbours two products of 448 * 448 cancel and six ones are left, so that a sum over cols is 6 / 8 of
    it; nothing of it is rounded in 8 bits (all scales are one), and sums of 32 bits hold it."""
    x, w = torch.ones(rows, cols), torch.ones(rows, cols)
    x[:, 0::8] = x[:, 1::8] = w[:, 0::8] = 448.0
    w[:, 1::8] = -448.0
    return x, w


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("rows", [1, 5, 16, 17, 40, 130])
def test_sums_of_32_bits_without_asking(X, rows, dtype):
    """Results whose own rounding would not cover what the 8-bit instruction drops."""
    x, w = cancelling(rows, 256)[0].to(dtype).cuda(), cancelling(70, 256)[1].cuda()
    assert (X.linear(x, X.quantize_weights(w)) == 192.0).all()
    y, kept = X.linear(x, X.quantize_weights(w), train=True)
    assert (y == 192.0).all()
    # the gradient of x: d_out against w's columns
    d, turned = cancelling(rows, 256)[0].to(dtype).cuda(), cancelling(70, 256)[1].t().contiguous().cuda()
    _, kept = X.linear(torch.ones((rows, 70), dtype=dtype, device="cuda"), X.quantize_weights(turned), train=True)
    d_x, _ = X.linear_backward(d, kept, X.quantize_weights(turned, turned=True))
    assert d_x.dtype == dtype and (d_x == 192.0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 16, 17, 200])
def test_experts_sum_in_32_bits_without_asking(X, T, dtype):
    x, w = cancelling(T, 256)[0].to(dtype).cuda(), cancelling(3 * 70, 256)[1].view(3, 70, 256).cuda()
    ids = torch.arange(2 * T, dtype=torch.int32).view(T, 2).remainder(3).cuda()
    weights = torch.full((T, 2), 0.5, device="cuda")
    q = X.quantize_weights(w)
    assert (X.experts(x, ids, weights, q) == 192.0).all()
    assert (X.experts(x, ids, weights, q, train=True)[0] == 192.0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,E,N,K", [(17, 2, 3, 257, 129), (300, 4, 8, 320, 640), (2100, 2, 5, 300, 512), (64, 5, 100, 200, 400)])
def test_training_and_evaluation_give_the_same(X, T, k, E, N, K, dtype):
    """(Up to 16 rows evaluation has a launch of its own, which adds in another order.)"""
    ids, w = routed(T, k, E, T, skew=True, empty=True)
    x, q = data(T, K, 1, dtype).cuda(), X.quantize_weights(weights_of(E, N, K, 2).cuda())
    for exact in (None, False, True):
        assert torch.equal(X.experts(x, ids.cuda(), w.cuda(), q, exact=exact), X.experts(x, ids.cuda(), w.cuda(), q, train=True, exact=exact)[0])
    one = X.quantize_weights(data(N, K, 3).cuda())
    for exact in (None, False, True):
        assert torch.equal(X.linear(x, one, exact=exact), X.linear(x, one, train=True, exact=exact)[0])


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [5, 33, 300])
def test_callers_choose(X, rows, dtype, exact):
    """linear, experts and both gradients of x with either sum, against 64 bits."""
    x, d, w = data(rows, 300, 1, dtype), data(rows, 130, 2, dtype), data(130, 300, 3)
    A, D, W = R.rounded(x.float()), R.rounded(d.float()), R.from_squares(*R.to_squares(w))[:, :300]
    q, t = X.quantize_weights(w.cuda()), X.quantize_weights(w.cuda(), turned=True)
    y, kept = X.linear(x.cuda(), q, train=True, exact=exact)
    d_x, _ = X.linear_backward(d.cuda(), kept, t, exact=exact)
    ids, ones = torch.zeros((rows, 1), dtype=torch.int32, device="cuda"), torch.ones((rows, 1), device="cuda")
    of_one, held = X.experts(x.cuda(), ids, ones, q, train=True, exact=exact)
    d_one, _, _ = X.experts_backward(d.cuda(), held, t, exact=exact)
    for got, a, b in ((y, A, W), (X.linear(x.cuda(), q, exact=exact), A, W), (of_one, A, W), (X.experts(x.cuda(), ids, ones, q, exact=exact), A, W),
                      (d_x, D, W.t().contiguous()), (d_one, D, W.t().contiguous())):
        want = a @ b.t()
        assert got.dtype == dtype and ((got.cpu().double() - want).abs() <= bounds(a, b, exact, dtype, want) + 4 * R.U * want.abs()).all()


def test_what_the_8_bit_instruction_costs(X):
    """The figures that callers choose by: the root mean square of the error over that of the result."""
    g = torch.Generator().manual_seed(11)
    for octaves, most in ((0, 2e-5), (6, 1e-4)):
        x, w = (torch.randn(n, 2048, generator=g) * torch.exp2((torch.rand(n, 2048, generator=g) - 0.5) * octaves) for n in (512, 512))
        want = R.rounded(x) @ R.from_squares(*R.to_squares(w)).t()
        a, b = X.quantize(x.cuda()), X.quantize_weights(w.cuda())
        for exact, limit in ((False, most), (True, 2e-7)):
            off = X.product(a, b, torch.float32, exact=exact).cpu().double() - want
            assert off.square().mean().sqrt() <= limit * want.square().mean().sqrt()


def test_weights_that_changed_since(X):
    """The weights are kept, not copied: gradients from others than the result was formed with are refused."""
    ids, w = routed(40, 2, 3, 1)
    x, d, mats = data(40, 100, 1).cuda(), data(40, 60, 2).cuda(), weights_of(3, 60, 100, 3).cuda()
    q, t, w = X.quantize_weights(mats), X.quantize_weights(mats, turned=True), w.cuda()
    _, kept = X.experts(x, ids.cuda(), w, q, train=True)
    first = X.experts_backward(d, kept, t)
    assert all(torch.equal(a, b) for a, b in zip(first, X.experts_backward(d, kept, t)))
    w *= 2
    with pytest.raises(ValueError, match="changed"):
        X.experts_backward(d, kept, t)
    with torch.inference_mode():
        v = w.clone()
        _, kept = X.experts(x, ids.cuda(), v, q, train=True)
        assert len(X.experts_backward(d, kept, t)) == 3
