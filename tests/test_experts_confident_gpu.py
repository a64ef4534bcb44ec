"""The gradient of routing where a router is confident: scores next to one or far below the smallest normal number.  References are formed
without differences that cancel, and bounds are relative to the gradient itself."""
import pytest
import torch

from tests import experts_rules as R
from tests.test_experts_route_gpu import rule_of

pytestmark = pytest.mark.gpu
TYPES = [(torch.float32, 0.0), (torch.bfloat16, 2.0 ** -8)]


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; there is no CPU fallback")
    from paper_1505_04956_amd import experts
    return experts


def gradient(X, l, rule, ids, dw):
    return torch.gather(X.route_backward(l.cuda(), rule, ids.cuda(), dw.cuda()).cpu().double(), 1, ids.long())


@pytest.mark.parametrize("dtype,rest", TYPES)
@pytest.mark.parametrize("low,high", [(8.0, 30.0), (-30.0, -8.0), (-3.0, 17.0)])
def test_sigmoid(X, low, high, dtype, rest):
    """dl = c dw s(l) s(-l): two exponentials, two additions, two divisions and three products, a rounding or two each."""
    g = torch.Generator().manual_seed(1)
    l = (low + (high - low) * torch.rand(40, 100, generator=g)).to(dtype)
    rule, dw = rule_of(X, 6, "sigmoid", renormalize=False, scale=2.5), torch.randn(40, 6, generator=g)
    ids = X.route(l.cuda(), rule)[0].cpu()
    at = torch.gather(l.double(), 1, ids.long())
    want = 2.5 * dw.double() * torch.sigmoid(at) * torch.sigmoid(-at)
    assert ((gradient(X, l, rule, ids, dw) - want).abs() <= (16 * 2 * R.U + rest) * want.abs()).all()


def share_of(l, ids, score):
    """[T, k] shares of the chosen in 64 bits, which add up to one."""
    at = torch.gather(l.double(), 1, ids.long())
    if score == "softmax":
        return torch.softmax(at, 1)
    s = torch.sigmoid(at)
    return s / s.sum(1, keepdim=True)


@pytest.mark.parametrize("dtype,rest", TYPES)
def test_sigmoid_renormalised_far_below(X, dtype, rest):
    """Scores of 1e-38 and less, whose shares are ordinary numbers: so is the gradient, c share s(-l) (dw - sum of share dw).  A score as small
    is a multiple of 2^-149, 6 more roundings at 3e-39."""
    g = torch.Generator().manual_seed(2)
    l = (-88.5 + 1.5 * torch.rand(40, 100, generator=g)).to(dtype)
    rule, dw = rule_of(X, 4, "sigmoid", scale=2.0), 300.0 * torch.randn(40, 4, generator=g)
    ids = X.route(l.cuda(), rule)[0].cpu()
    p, d = share_of(l, ids, "sigmoid"), dw.double()
    want = 2.0 * p * torch.sigmoid(-torch.gather(l.double(), 1, ids.long())) * (d - (p * d).sum(1, keepdim=True))
    # every share is off by 24 roundings (exponential at 88, sum, division, the score's own), and by as many what they weigh
    size = 2.0 * p * (d.abs() + (p * d.abs()).sum(1, keepdim=True))
    assert ((gradient(X, l, rule, ids, dw) - want).abs() <= 2 * 32 * 2 * R.U * size + rest * want.abs()).all()
