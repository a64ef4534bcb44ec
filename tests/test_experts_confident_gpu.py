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
