"""The norm of many gradients and clipping by it on the GPU, against 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
STEP = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}      # between the smallest numbers


@pytest.fixture(scope="module")
def G():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; there is no CPU fallback")
    from paper_1505_04956_amd import gradients
    return gradients


def exact_norm(tensors):
    return math.sqrt(math.fsum(float((t.detach().cpu().double() ** 2).sum()) for t in tensors))


def near(got, want):
    """One rounding to 32 bits, and 64-bit sums."""
    return abs(got - want) <= want * (2.0 ** -24 + 1e-12) + 2.0 ** -149


def check(got, grad, factor):
    """The factor and the product are each rounded to 32 bits, the result to its type."""
    want = grad.cpu().double() * factor
    allowed = want.abs() * (2.0 ** -24 * 2.1 + HALF[got.dtype] * 1.01) + STEP[got.dtype] / 2 + 2.0 ** -149
    assert ((got.cpu().double() - want).abs() <= allowed).all()


def make(sizes, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    flat = (torch.randn(sum(sizes) + 7, generator=g) * scale).to(dtype).cuda()
    return list(flat[3:3 + sum(sizes)].split(sizes))


SETS = [[1], [4096], [4097], [13, 0, 5000, 1, 7], [8192, 4096, 0, 0], [0, 0, 3], [16 * 24 * 32, 24 * 32, 16 * 32], [3] * 64, [5, 4099] * 33, [1] * 200, [100_003, 17, 2_000_001],
        [12345] * 130]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", SETS, ids=lambda s: "%dx%d" % (len(s), sum(s)))
def test_norm_and_clip(G, sizes, dtype):
    grads = make(sizes, dtype, len(sizes))
    want = exact_norm(grads)
    assert near(G.norm(grads).item(), want)
    again = G.norm(grads)
    assert torch.equal(again, G.norm(grads)) and again.shape == () and again.dtype == torch.float32
    for out_type in TYPES:
        for limit in (want * 0.3, want * 2):
            flat = torch.full((sum(sizes) + 9,), 5.0, dtype=out_type, device="cuda")
            out = list(flat[5:5 + sum(sizes)].split(sizes))
            was = [t.clone() for t in grads]
            assert near(G.clip(grads, limit, out=out).item(), want)
            assert all(torch.equal(a, b) for a, b in zip(grads, was))
            assert (flat[:5] == 5.0).all() and (flat[5 + sum(sizes):] == 5.0).all()
            for a, b in zip(out, grads):
                check(a, b, min(1.0, limit / want))
    was = [t.clone() for t in grads]
    G.clip(grads, want * 1.5)
    assert all(torch.equal(a, b) for a, b in zip(grads, was))
    G.clip(grads, want * 0.25)
    for a, b in zip(grads, was):
        check(a, b, 0.25)


def test_types_together(G):
    grads = make([1000, 5000], torch.float32, 1) + make([3, 9000], torch.bfloat16, 2) + make([77, 4096], torch.float16, 3)
    want, was = exact_norm(grads), [t.clone() for t in grads]
    out = [torch.empty_like(t, dtype=d) for t, d in zip(grads, (torch.bfloat16, torch.float32, torch.float16, torch.float32, torch.float32, torch.bfloat16))]
    out[2] = grads[2]                                             # one of them in place
    assert near(G.clip(grads, 1.0, out=out).item(), want)
    for n, (a, b) in enumerate(zip(out, was)):
        check(a, b, 1.0 / want)
        assert n == 2 or torch.equal(grads[n], b)
    grads[2].copy_(was[2])
    G.clip(grads, want * 3, out=out)
    assert all(torch.equal(a, b.to(a.dtype)) for a, b in zip(out, was))


def test_numbers_at_the_edge(G):
    """Squares beyond 32 bits at either end; what is no finite number; a limit of zero."""
    big, small = [torch.full((5000,), 1e30, device="cuda")], [torch.full((5000,), 1e-30, device="cuda")]
    assert near(G.norm(big).item(), exact_norm(big)) and near(G.norm(small).item(), exact_norm(small))
    zeros = [torch.zeros(100, device="cuda")]
    assert G.clip(zeros, 0.0).item() == 0.0 and (zeros[0] == 0).all()
    g = [torch.ones(100, device="cuda"), torch.full((3,), -2.0, device="cuda")]
    assert G.clip(g, 0.0).item() == pytest.approx(math.sqrt(112)) and all((t == 0).all() for t in g)
    g = [torch.ones(100, device="cuda"), torch.tensor([1.0, float("nan")], device="cuda")]
    assert math.isnan(G.norm(g).item()) and math.isnan(G.clip(g, 1.0).item()) and all(torch.isnan(t).all() for t in g)
    g = [torch.ones(5000, device="cuda"), torch.tensor([1.0, float("inf")], device="cuda")]
    assert math.isinf(G.norm(g).item()) and math.isinf(G.clip(g, 1.0).item())
    assert (g[0] == 0).all() and g[1][0] == 0 and torch.isnan(g[1][1])
    g = [torch.tensor([1.0, float("inf")], device="cuda")]
    assert math.isinf(G.clip(g, float("inf")).item()) and g[0][0] == 1.0 and math.isinf(g[0][1].item())
    assert math.isinf(G.norm([torch.full((4,), 3e38, device="cuda")]).item())           # (the norm itself is beyond 32 bits)
    nothing = [torch.empty(0, device="cuda")]
    assert G.norm(nothing).item() == 0.0 and G.clip(nothing, 1.0).item() == 0.0


def test_runs_that_share_memory_are_refused(G):
    from paper_1505_04956_amd.binding import AsgdError
    flat = torch.randn(1000, device="cuda")
    was = flat.clone()
    other = torch.empty(1000, device="cuda")
    for grads, out in (([flat, flat], None), ([flat[:600], flat[500:]], None), ([flat[:500], flat[500:]], [other[:500], other[400:900]]),
                       ([flat[:500], flat[500:]], [flat[500:], flat[:500]]), ([flat[:400]], [flat[1:401]]),
                       ([flat[:500]], [flat.view(torch.bfloat16)[:500]])):
        with pytest.raises(AsgdError):
            G.clip(grads, 1.0, out=out)
    torch.cuda.synchronize()
    assert torch.equal(flat, was)
    assert G.norm([flat, flat]).item() == pytest.approx(math.sqrt(2) * flat.double().norm().item(), rel=1e-6)     # (they are only read)
    G.clip([flat[500:], flat[:500]], 1.0)
    assert flat.double().norm().item() == pytest.approx(1.0, rel=1e-6)


def test_streams_and_graphs(G):
    sizes = [5000, 3, 70_000]
    grads, out = make(sizes, torch.bfloat16, 1), make(sizes, torch.float32, 2)
    many = make([100] * 90, torch.float32, 3)
    source, source_many = [t.clone() for t in grads], [t.clone() for t in many]
    graphs, held = [], []
    for call in (lambda: G.clip(grads, 1.0, out=out), lambda: G.clip(many, 2.0)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            held.append(call())
    side = torch.cuda.Stream()
    for n in range(3):
        for t, s in zip(grads, source):
            t.copy_(s * (n + 1))
        for t, s in zip(many, source_many):
            t.copy_(s * (n + 1))
        want, want_many = exact_norm(grads), exact_norm(many)
        before = [t.clone() for t in many]
        for h in held:
            h.zero_()
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        eager = G.norm(grads)
        torch.cuda.synchronize()
        assert near(held[0].item(), want) and near(held[1].item(), want_many) and torch.equal(eager, held[0])
        for a, b in zip(out, grads):
            check(a, b, min(1.0, 1.0 / want))
        for a, b in zip(many, before):
            check(a, b, min(1.0, 2.0 / want_many))


def test_more_than_two_to_the_32_bytes(G):
    """Places in a long run pass 32 bits."""
    n = (1 << 31) + 5000
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-3:] = torch.tensor([3.0, 0.0, 4.0])
    g[5] = 12.0
    assert G.clip([g], 6.5).item() == 13.0
    assert g[5] == 6.0 and g[-3] == 1.5 and g[-1] == 2.0 and g[-2] == 0.0 and (g != 0).sum() == 3


def test_what_is_clipped_counts_as_modified(G):
    """A backward pass through what was clipped after it was saved is refused, as after an operation of torch in place: autograd's, and experts_backward()'s."""
    from paper_1505_04956_amd import experts as X
    a, b = torch.ones(5000, device="cuda", requires_grad=True), torch.ones(5000, device="cuda")
    y, z = (a * b).sum(), (a * b).sum()
    out, was = torch.empty_like(b), b._version
    G.norm([b]), G.clip([b], 1.0, out=[out])
    z.backward()                                                    # (it was only read)
    assert out._version > 0 and b._version == was and (a.grad == 1).all()
    G.clip([b], 1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    w = torch.randn(3, 20, 40, device="cuda")
    x = torch.randn(7, 40, device="cuda")
    ids, weights = X.route(torch.randn(7, 3, device="cuda"), X.Rule(2))
    got, kept = X.experts(x, ids, weights, X.quantize_weights(w), train=True)
    G.clip([weights], 0.5)
    with pytest.raises(ValueError, match="have changed"):
        X.experts_backward(got, kept, X.quantize_weights(w, turned=True))


@pytest.mark.parametrize("n", [1000, 100_000])
def test_runs_that_are_only_read_may_share_memory(G, n):
    """The same gradient twice, and views that overlap, into memory of their own: each counts as often as it is listed."""
    flat = make([n], torch.float32, n)[0]
    was = flat.clone()
    for grads in ([flat, flat], [flat[:n // 2], flat[n // 3:], flat], [flat[n // 2:], flat[:n // 2 + 3]]):
        want, out = exact_norm(grads), [torch.empty_like(t, dtype=d) for t, d in zip(grads, TYPES)]
        assert near(G.clip(grads, want * 0.3, out=out).item(), want)
        for a, b in zip(out, grads):
            check(a, b, 0.3)
    assert torch.equal(flat, was)
