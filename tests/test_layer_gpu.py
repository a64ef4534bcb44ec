"""A whole layer of experts for few rows on the GPU, against 64 bits; and the calls of experts, 4 bits, layers and gradients together."""
import pytest
import torch

from tests import experts_rules as R
from tests import micro_rules as Q

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ROUNDING = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 6e-8}


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; there is no CPU fallback")
    from paper_1505_04956_amd import layer
    return layer


def make(L, T, E, D, H, N, bits, dtype, seed):
    """(x, logits, up, down, their matrices in 64 bits)"""
    from paper_1505_04956_amd import experts as X, micro as M
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(T, D, generator=g) * torch.exp(torch.randn(D, generator=g) * 0.5)).to(dtype)
    logits = torch.randn(T, E, generator=g) * 2
    up, down = torch.randn(E, 2 * H, D, generator=g) / D ** 0.5, torch.randn(E, N, H, generator=g) / H ** 0.5
    if bits == 4:
        mu, md = M.quantize(up.cuda()), M.quantize(down.cuda())
        return x, logits, mu, md, Q.matrix_of(mu), Q.matrix_of(md)
    mu, md = X.quantize_weights(up.cuda()), X.quantize_weights(down.cuda())
    of = lambda m: torch.stack([R.from_squares(v, s)[:, :m.cols] for v, s in zip(m.values.cpu(), m.scales.cpu())])  # noqa: E731
    return x, logits, mu, md, of(mu), of(md)


def close(got, want, bound, dtype):
    off = (got.cpu().double() - want).abs()
    allowed = bound + ROUNDING[dtype] * (want.abs() + bound) + SMALLEST[dtype]
    assert (off <= allowed).all(), float((off / allowed).max())


SHAPES = [(1, 8, 2, 64, 32, 48), (1, 64, 6, 300, 200, 130), (2, 5, 5, 257, 129, 100), (5, 100, 5, 100, 70, 33), (15, 9, 2, 513, 260, 17), (16, 40, 3, 128, 128, 256),
          (16, 7, 7, 1000, 40, 1), (3, 300, 8, 33, 1, 20), (1, 1, 1, 1, 1, 1), (4, 1024, 20, 40, 24, 16), (2, 64, 64, 40, 24, 16), (16, 1000, 3, 50, 24, 16), (8, 256, 8, 100, 300, 40), (7, 33, 2, 5000, 20, 30), (1, 200, 3, 9000, 33, 40), (8, 12, 2, 600, 100, 70)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k,D,H,N", SHAPES)
def test_layers(L, T, E, k, D, H, N, dtype, bits):
    from paper_1505_04956_amd import experts as X
    x, logits, up, down, u64, d64 = make(L, T, E, D, H, N, bits, dtype, T * E + D)
    gelu = (T + E + D) % 2 == 1
    rule = X.Rule(k, score=X.SIGMOID if T % 2 else X.SOFTMAX, scale=1.5, renormalize=D % 2 == 0)
    bias = (torch.randn(E, generator=torch.Generator().manual_seed(E)) * 0.1).cuda() if T % 2 else None
    if T > 2:
        logits[1] = -float("inf")
        logits[2, 1:] = -float("inf")
    y, ids, weights = L.layer(x.cuda(), logits.cuda(), rule, up, down, bias=bias, activation=L.GELU if gelu else L.SILU)
    i2, w2 = X.route(logits.cuda(), rule, bias=bias)
    assert torch.equal(ids, i2) and torch.equal(weights, w2) and y.dtype == dtype and y.shape == (T, N)
    if T > 2:
        assert (ids[1] == -1).all() and (y[1] == 0).all() and (ids[2, 0] == 0) and (ids[2, 1:] == -1).all()
    want, bound = Q.layer(x.float(), ids.cpu(), weights.cpu(), u64, d64, bits, gelu)
    close(y, want, bound, dtype)


@pytest.mark.parametrize("bits", [8, 4])
def test_logits_of_every_type_and_strides(L, bits):
    from paper_1505_04956_amd import experts as X
    x, logits, up, down, _, _ = make(L, 6, 12, 100, 40, 30, bits, torch.float16, 1)
    wide_x, wide_l = torch.full((6, 300), 9.0, dtype=torch.float16).cuda(), torch.full((12, 31), 50.0).cuda()
    wide_x[:, 5:105], wide_l[::2, 3:15] = x.cuda(), logits.cuda()
    rule = X.Rule(3)
    want = L.layer(x.cuda(), logits.cuda(), rule, up, down)
    got = L.layer(wide_x[:, 5:105], wide_l[::2, 3:15], rule, up, down)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for dtype in (torch.bfloat16, torch.float16):
        l = logits.to(dtype).cuda()
        got, want = L.layer(x.cuda(), l, rule, up, down), L.layer(x.cuda(), l.float(), rule, up, down)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("bits", [8, 4])
def test_what_is_not_a_number_stays_with_its_rows(L, bits):
    from paper_1505_04956_amd import experts as X
    x, logits, up, down, _, _ = make(L, 7, 6, 300, 140, 50, bits, torch.float32, 2)
    rule = X.Rule(2)
    want, ids, _ = L.layer(x.cuda(), logits.cuda(), rule, up, down)
    bad = x.clone()
    bad[1, 17], bad[4, 299] = float("nan"), float("inf")
    y, _, _ = L.layer(bad.cuda(), logits.cuda(), rule, up, down)
    others = [0, 2, 3, 5, 6]
    assert torch.isnan(y[[1, 4]]).all() and torch.equal(y[others], want[others])
    # scales of one expert's weights
    for m in (up, down):
        kept = m.scales.clone()
        if bits == 4:
            m.scales[3, 0, 0] = 255
        else:
            m.scales[3, 0, 0] = float("nan")
        y, _, _ = L.layer(x.cuda(), logits.cuda(), rule, up, down)
        goes = (ids == 3).any(1)
        assert goes.any() and not goes.all()
        assert torch.isnan(y[goes]).any(1).all() and torch.equal(y[~goes], want[~goes])
        m.scales.copy_(kept)
    # a logit
    bad = logits.clone()
    bad[2, 3] = float("nan")
    y, i, w = L.layer(x.cuda(), bad.cuda(), rule, up, down)
    assert torch.isnan(w[2][i[2] >= 0]).all() and torch.isnan(y[2]).all() and torch.equal(y[[0, 1, 3, 4, 5, 6]], want[[0, 1, 3, 4, 5, 6]])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("T", [1, 5, 16])
def test_the_same_as_the_calls_that_it_stands_for(L, T, bits):
    from paper_1505_04956_amd import experts as X, micro as M
    D, H, N, E, k = 200, 96, 70, 6, 2
    x, logits, up, down, _, _ = make(L, T, E, D, H, N, bits, torch.float32, 3)
    rule = X.Rule(k)
    y, ids, weights = L.layer(x.cuda(), logits.cuda(), rule, up, down)
    order = X.plan(ids, E)
    P = M if bits == 4 else X
    u = P.product(P.quantize(x.cuda()), up, torch.float32, order, gather=True)
    h = torch.nn.functional.silu(u[:, :H]) * u[:, H:]
    z = X.experts_sum(P.product(P.quantize(h), down, torch.float32, order), order, torch.float32, weights)
    # a value of h next to a border may be rounded the other way: one of 96, by a step of at most a quarter of it
    assert ((y - z).norm(dim=1) <= 0.05 * z.norm(dim=1)).all() and (y - z).norm() <= 0.02 * z.norm()


def test_no_rows(L):
    from paper_1505_04956_amd import experts as X
    x, logits, up, down, _, _ = make(L, 1, 6, 100, 40, 30, 8, torch.float32, 1)
    y, ids, weights = L.layer(x[:0].cuda(), logits[:0].cuda(), X.Rule(2), up, down)
    assert y.shape == (0, 30) and ids.shape == weights.shape == (0, 2)


@pytest.mark.parametrize("bits", [8, 4])
def test_two_streams_and_graphs(L, bits):
    """Two captured calls and an eager one, each with scratch of its own, on streams of their own."""
    from paper_1505_04956_amd import experts as X
    x, logits, up, down, _, _ = make(L, 16, 20, 300, 128, 90, bits, torch.bfloat16, 4)
    x, logits, rule = x.cuda(), logits.cuda(), X.Rule(4, score=X.SIGMOID)
    a, b = (x[:9].clone(), logits[:9].clone()), (x[9:].clone(), logits[9:].clone())
    want = [[t.clone() for t in L.layer(*c, rule, up, down)] for c in (a, b)]
    graphs, held = [], []
    for c in (a, b):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            held.append(L.layer(*c, rule, up, down))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for n in range(3):
        for h in held:
            for t in h:
                t.zero_()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        eager = L.layer(*a, rule, up, down)
        torch.cuda.synchronize()
        for h, w in zip(held + [eager], want + want[:1]):
            assert all(torch.equal(p, q) for p, q in zip(h, w))


def test_trained_with_clipped_gradients_then_served(L):
    """As the calls are used: experts are trained in 8 bits with clipped gradients, brought to 4 bits, and serve prompts and single rows; and
    a layer of two matrices made of them serves a few rows."""
    from paper_1505_04956_amd import experts as X, gradients as G, micro as M
    g = torch.Generator().manual_seed(5)
    T, E, D, N, k = 400, 6, 96, 80, 2
    x, logits = torch.randn(T, D, generator=g).bfloat16().cuda(), torch.randn(T, E, generator=g).cuda()
    w, target = (torch.randn(E, N, D, generator=g) / D ** 0.5).cuda(), torch.randn(T, N, generator=g).cuda()
    rule = X.Rule(k)
    ids, weights = X.route(logits, rule)
    for _ in range(3):
        y, kept = X.experts(x, ids, weights, X.quantize_weights(w), train=True)
        d_y = ((y.float() - target) / T).bfloat16()
        _, d_w, d_weights = X.experts_backward(d_y, kept, X.quantize_weights(w, turned=True))
        d_logits = X.route_backward(logits, rule, ids, d_weights)
        plain = torch.sqrt((d_w.double() ** 2).sum() + (d_logits.double() ** 2).sum())
        was, limit = [d_w.clone(), d_logits.clone()], float(plain) / 3
        norm = G.clip([d_w, d_logits], limit)
        assert abs(norm.item() - plain.item()) <= 1e-6 * plain.item()
        for a, b in zip((d_w, d_logits), was):
            assert (a.double() - b.double() * (limit / plain)).abs().max() <= 3e-7 * b.abs().max()
        w -= 0.1 * d_w
    small = M.quantize(w)
    many = M.experts(x, ids, weights, small)
    few = M.experts(x[:10], ids[:10], weights[:10], small)
    v = M.expand(small).cpu().double()
    q = Q.four(x[:10].cpu().float())
    c = weights[:10].cpu().double()
    want = torch.stack([sum(c[t, j] * (v[ids[t, j]] @ q[t]) for j in range(k)) for t in range(10)])
    for got in (many[:10], few):
        assert (got.cpu().double() - want).abs().max() <= 2.0 ** -8 * want.abs().max() + 1e-5
    up = M.quantize(torch.cat([w, w], 1).contiguous())                    # h = f(w x) * w x
    down = M.quantize(w.transpose(1, 2).contiguous())
    y, i, c = L.layer(x[:10], logits[:10], rule, up, down)
    assert torch.equal(i, ids[:10]) and torch.equal(c, weights[:10])
    want, bound = Q.layer(x[:10].cpu().float(), i.cpu(), c.cpu(), Q.matrix_of(up), Q.matrix_of(down), 4, False)
    close(y, want, bound, torch.bfloat16)


@pytest.mark.parametrize("shared", [False, True])
def test_the_example_clips_its_gradients_and_serves_in_four_bits(L, shared):
    """A step with a limit moves by the gradients of one without, all scaled alike; the maps in 4 bits are applied as experts() and linear() do."""
    from paper_1505_04956_amd import clusterwise as C, experts as X, micro as M
    g = torch.Generator().manual_seed(1)
    k, d, n, rows, rate = 5, 40, 24, 600, 0.05
    x, target = torch.randn(rows, d, generator=g).cuda(), torch.randn(rows, n, generator=g).cuda()
    centroids = torch.randn(k, d, generator=g).cuda()
    make = lambda: C.ClusterwiseLinear(centroids.clone(), n, shared=shared)  # noqa: E731
    parts = lambda m: [t for t in (m.w, m.centroids, m.shared) if t is not None]  # noqa: E731
    free, bound, far = make(), make(), make()
    start = [t.clone() for t in parts(free)]
    losses = [m.step(x, target, rate, limit).item() for m, limit in ((free, None), (bound, 0.01), (far, 1e6))]
    assert losses[0] == losses[1] == losses[2]
    assert all(torch.equal(a, b) for a, b in zip(parts(free), parts(far)))
    rates = [rate, rate, rate * 2 / k]
    moved = [[(a.double() - b.double()) / r for a, b, r in zip(start, parts(m), rates)] for m in (free, bound)]
    norm = [sum(float((t ** 2).sum()) for t in m) ** 0.5 for m in moved]
    # (what a step moves by is rounded to the weights' last bit: 2^-24 of weights up to 8, over the rate)
    count = sum(t.numel() for t in start)
    slack = 2.0 ** -24 * 8 / (rate * 2 / k) * count ** 0.5
    assert norm[0] > 0.1 and abs(norm[1] - 0.01) <= slack
    for a, b in zip(*moved):
        assert (b - a * (0.01 / norm[0])).abs().max() <= 2 * slack
    served = free.small()
    y = served(x)
    ids, weights = X.route(free.logits(x), free.rule)
    want = M.experts(x.bfloat16(), ids, weights, M.quantize(free.w))
    if shared:
        want = want.float() + M.linear(x.bfloat16(), M.quantize(free.shared)).float()
    assert torch.equal(y, want) and torch.equal(served(x[:3]).float(), served(x[:3]).float()) and y.shape == (rows, n)
    said = []
    got, _ = C.run(samples=60_000, steps=2, k=4, batch=1000, shared=shared, limit=0.5, small=lambda *l: said.extend(l))
    assert len(got) == 2 and len(said) == 2 and all(0 < v < 1e9 for v in got + said)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("T", [3, 12])
@pytest.mark.parametrize("low", [-3.0, -5.0, -6.5, -9.0, -11.0])
def test_gates_far_below_zero(L, monkeypatch, low, T, bits):
    """g / 2 * (1 + erf(g / sqrt(2))) where the two all but cancel: h keeps its digits, and blocks of such h are not lost.  For g < 0, |f'(g)| is at most
    (|g| + 1) |f(g)| (Mills' ratio); the argument of the error function is within 2 units of 2^-24, the function within 16 of its last place, and there are
    two products more."""
    from paper_1505_04956_amd import experts as X, micro as M

    def activated(g, u, gelu):
        assert gelu and (g < 0).all()
        return 0.5 * g * torch.special.erfc(-g / 2 ** 0.5) * u

    def bound(g, u, dg, du, gelu):
        f = activated(g, torch.ones_like(u), gelu).abs()
        assert ((g.abs() + 1) * dg < 0.1).all()                     # (e^0.1 < 1.11: what the second order adds)
        return f * ((g.abs() + 1) * (dg + 2 * Q.U * g.abs()) * 1.11 + 40 * Q.U) * (u.abs() + du) + f * du + 2 * Q.U * f * u.abs() + 1e-37
    monkeypatch.setattr(Q, "activated", activated)
    monkeypatch.setattr(Q, "activated_bound", bound)
    E, D, H, N = 3, 64, 97, 40
    g = torch.Generator().manual_seed(int(-10 * low) + T)
    rand = lambda *shape: torch.rand(*shape, generator=g)  # noqa: E731
    x, logits = 0.9 + 0.2 * rand(T, D), torch.randn(T, E, generator=g)
    up = torch.cat([(low - 0.5 * rand(E, H, 1)) / D * (0.9 + 0.2 * rand(E, H, D)), (0.5 + rand(E, H, D)) / D], 1)
    down = torch.randn(E, N, H, generator=g) / H ** 0.5
    of = M.quantize if bits == 4 else X.quantize_weights
    up, down = of(up.cuda()), of(down.cuda())
    full = lambda m: Q.matrix_of(m) if bits == 4 else torch.stack([R.from_squares(v, s)[:, :m.cols] for v, s in zip(m.values.cpu(), m.scales.cpu())])  # noqa: E731
    y, ids, weights = L.layer(x.cuda(), logits.cuda(), X.Rule(2), up, down, activation=L.GELU)
    want, off = Q.layer(x, ids.cpu(), weights.cpu(), full(up), full(down), bits, True)
    # (what may be off is a small part of what is there, so the test says something)
    assert off.norm() < 0.1 * want.norm()
    close(y, want, off, torch.float32)


# (rows, experts, groups): routed in the first product's launch, and by one of its own; groups of whole lanes and others, all widths of a lane
GROUPS = [(5, 60, 6), (8, 64, 8), (3, 128, 4), (2, 256, 8), (8, 250, 5), (16, 60, 6), (16, 64, 8), (9, 128, 4), (16, 250, 5), (16, 256, 8), (16, 512, 16), (3, 300, 10), (7, 512, 64), (16, 1000, 10), (16, 1024, 64),
          (2, 1001, 7), (1, 1024, 16)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,groups", GROUPS)
def test_groups_scores_and_logits_of_every_type(L, T, E, groups, dtype):
    """In both launches that route: the choice and the weights are route()'s bit for bit, whatever the rule, the logits' type and how they lie."""
    from paper_1505_04956_amd import experts as X
    D, H, N = 40, 24, 16
    for n, (score, by, with_bias, renormalize) in enumerate([(X.SOFTMAX, X.BEST, False, True), (X.SIGMOID, X.BEST_TWO, True, True), (X.SOFTMAX, X.BEST_TWO, True, False),
                                                             (X.SOFTMAX, X.BEST_TWO, False, True), (X.SIGMOID, X.BEST, False, False), (X.SOFTMAX, X.BEST, True, True)]):
        bits = 4 if (n + E) % 2 else 8
        x, logits, up, down, u64, d64 = make(L, T, E, D, H, N, bits, torch.float32, E + n)
        apart = torch.zeros(T, E + 9, dtype=dtype, device="cuda")
        l = apart[:, n % 3:n % 3 + E]                               # rows that begin anywhere, and aligned ones
        l.copy_(logits)
        if T > 2:
            l[1] = -float("inf")
            l[2, E // groups:] = -float("inf")                      # one group left, and fewer experts than are chosen of it
            l[2, 3:] = -float("inf")
        bias = (torch.randn(E, generator=torch.Generator().manual_seed(n)) * 0.2).cuda() if with_bias else None
        rule = X.Rule(4, score=score, groups=groups, kept=max(1, groups // 3), group_by=by, renormalize=renormalize, scale=2.0)
        for lay in (l, l.contiguous()):
            y, ids, weights = L.layer(x.cuda(), lay, rule, up, down, bias=bias)
            i2, w2 = X.route(lay, rule, bias=bias)
            assert torch.equal(ids, i2) and torch.equal(weights, w2)
        if T > 2:
            assert (ids[1] == -1).all() and (y[1] == 0).all() and (ids[2] >= 0).sum() == 3
        want, bound = Q.layer(x, ids.cpu(), weights.cpu(), u64, d64, bits, False)
        close(y, want, bound, torch.float32)


@pytest.mark.parametrize("T,E", [(6, 60), (6, 61), (16, 300), (16, 301), (16, 1000), (16, 1001)])
def test_sixteen_bit_logits_in_both_launches(L, T, E):
    from paper_1505_04956_amd import experts as X
    x, logits, up, down, _, _ = make(L, T, E, 64, 24, 20, 4, torch.bfloat16, T + E)
    for dtype in (torch.bfloat16, torch.float16):
        l = logits.to(dtype).cuda()
        got, want = L.layer(x.cuda(), l, X.Rule(5), up, down), L.layer(x.cuda(), l.float(), X.Rule(5), up, down)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("shared", [False, True])
def test_what_the_example_says_of_its_maps_in_four_bits(L, shared, monkeypatch):
    """The evaluation in 4 bits is that of the trained maps' 4-bit values, and the two losses that are said differ by no more than the two results do:
    |l4 - l8| <= sqrt(2 l8 m) + m / 2 with m the mean square of the difference (Cauchy and Schwarz), and what 32-bit means lose."""
    from paper_1505_04956_amd import clusterwise as C, experts as X
    held, said = {}, []
    small = C.ClusterwiseLinear.small

    def watched(self):
        served = small(self)

        def forward(x):
            held["x"], held["y8"], held["y4"], held["model"] = x, self.forward(x), served(x), self
            return held["y4"]
        return forward
    monkeypatch.setattr(C.ClusterwiseLinear, "small", watched)
    C.run(samples=60_000, steps=2, k=4, batch=1000, shared=shared, limit=0.5, small=lambda *l: said.extend(l))
    l8, l4 = said
    m = float((held["y4"].double() - held["y8"].double()).square().sum(1).mean())
    assert m > 0 and abs(l4 - l8) <= ((2 * l8 * m) ** 0.5 + m / 2) * (1 + 1e-3) + 1e-4 * l8
    model, x = held["model"], held["x"][:50]
    ids, weights = X.route(model.logits(held["x"]), model.rule)
    q, maps = Q.four(x.bfloat16().float().cpu()), [Q.four(w.cpu()) for w in model.w]
    y, mags = torch.zeros(50, maps[0].shape[0], dtype=torch.float64), torch.zeros(50, maps[0].shape[0], dtype=torch.float64)
    for t in range(50):
        for e, c in zip(ids[t].tolist(), weights[t].tolist()):
            y[t] += c * (maps[e] @ q[t])
            mags[t] += abs(c) * (maps[e].abs() @ q[t].abs())
    allowed = Q.product_bound(mags, x.shape[1]) + 2.0 ** -8 * y.abs() + 8 * Q.U * mags
    if shared:
        b = Q.four(model.shared.cpu())
        allowed += Q.product_bound(q.abs() @ b.abs().t(), x.shape[1]) + 2.0 ** -8 * (q @ b.t()).abs()
        y = y + q @ b.t()
        allowed += 2 * Q.U * y.abs()
    assert ((held["y4"][:50].cpu().double() - y).abs() <= 1.01 * allowed).all()


@pytest.mark.parametrize("shared", [False, True])
def test_the_examples_maps_in_four_bits_stay_what_they_were(L, shared):
    """What small() gave goes on giving the model of that moment, router and maps, while the model is trained on."""
    from paper_1505_04956_amd import clusterwise as C
    g = torch.Generator().manual_seed(2)
    x, target = torch.randn(300, 40, generator=g).cuda(), torch.randn(300, 24, generator=g).cuda()
    model = C.ClusterwiseLinear(torch.randn(5, 40, generator=g).cuda(), 24, shared=shared)
    served = model.small()
    was = served(x)
    for _ in range(3):
        model.step(x, target, 0.5)
    assert torch.equal(served(x), was) and not torch.equal(model.small()(x), was)
