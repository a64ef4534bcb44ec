"""Routing on the GPU against the definition in 64 bits: what is chosen, the weights, the gradient of the logits, the order."""
import math

import pytest
import torch

from tests import experts_rules as R

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; there is no CPU fallback")
    from paper_1505_04956_amd import experts
    return experts


def rule_of(X, k, score, groups=1, kept=1, two=False, renormalize=True, scale=1.0):
    return X.Rule(k, score=X.SOFTMAX if score == "softmax" else X.SIGMOID, groups=groups, kept=kept,
                  group_by=X.BEST_TWO if two else X.BEST, renormalize=renormalize, scale=scale)


def logits_of(T, E, seed, dtype=torch.float32, grid=8):
    """Multiples of 1 / grid between -6 and 6: many ties, and every type holds them."""
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, E, generator=g) * 1.5 * grid).round().clamp(-6 * grid, 6 * grid).div(grid).to(dtype)


def weight_bound(E):
    """Relative: the subtraction in the exponent (up to 12 units of |l| in half-ulps), exp (2), the sum over E (lanes, then six
    steps) and its terms (14 each), division, scale."""
    return (12 + 2 + E / 64 + 6 + 14 + 8) * 2 * R.U


SHAPES = [(1, 1, 1, 1, 1), (1, 64, 6, 1, 1), (3, 7, 7, 1, 1), (65, 65, 4, 5, 2), (130, 160, 6, 8, 3), (33, 256, 8, 8, 4), (9, 500, 12, 4, 4),
          (5, 1000, 32, 1, 1), (4, 1024, 64, 64, 64), (6, 1024, 9, 64, 1), (17, 128, 2, 64, 1), (2, 72, 40, 3, 2),
          (9, 1000, 3, 10, 2), (7, 512, 2, 1, 1)]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("T,E,k,groups,kept", SHAPES)
def test_choice_by_logits_and_weights(X, T, E, k, groups, kept, score, renormalize):
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        l = logits_of(T, E, T + E, dtype)
        ids, w = X.route(l.cuda(), rule_of(X, k, score, groups, kept, False, renormalize, 2.5))
        want = R.choose(l, score, None, k, groups, kept, False)
        assert torch.equal(ids.cpu(), want)                              # the keys are the logits: nothing is rounded
        ref = R.chosen_weights(l, score, None, want, renormalize, 2.5)
        assert ((w.cpu().double() - ref).abs() <= weight_bound(E) * ref + 1e-45).all()


@pytest.mark.parametrize("score,two", [("sigmoid", True), ("sigmoid", False), ("softmax", False), ("softmax", True)])
@pytest.mark.parametrize("T,E,k,groups,kept", [s for s in SHAPES if s[1] // s[3] >= 2])
def test_choice_with_a_bias(X, T, E, k, groups, kept, score, two):
    g = torch.Generator().manual_seed(E)
    l = torch.randn(T, E, generator=g) * 1.5
    bias = torch.randn(E, generator=g) * 0.1
    ids, w = X.route(l.cuda(), rule_of(X, k, score, groups, kept, two, True), bias=bias.cuda())
    ids = ids.cpu()
    # keys are rounded to 32 bits: whatever is chosen is as good as what the 64-bit keys would choose, to those roundings
    tie = weight_bound(E) + 8 * R.U
    key = R.keys(l, score, bias)
    value = R.group_values(l, score, bias, groups, two)
    of = (ids // (E // groups)).long()
    for t in range(T):
        row = ids[t].tolist()
        assert len(set(row)) == k and min(row) >= 0
        got = key[t, ids[t].long()]
        assert (got[:-1] >= got[1:] - tie).all()
        if len(set(of[t].tolist())) == kept:                              # (else the kept groups are not all visible)
            mine = torch.zeros(groups, dtype=torch.bool)
            mine[of[t]] = True
            if kept < groups:
                assert value[t][mine].min() >= value[t][~mine].max() - 2 * tie
            rest = key[t].clone()
            rest[ids[t].long()] = -INF
            rest[~mine.repeat_interleave(E // groups)] = -INF
            assert got.min() >= rest.max() - tie
    ref = R.chosen_weights(l, score, bias, ids, True, 1.0)
    assert ((w.cpu().double() - ref).abs() <= weight_bound(E) * ref + 1e-45).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
def test_masked_experts_and_rows(X, score, renormalize):
    l = logits_of(8, 100, 5)
    l[0] = -INF                                     # a row without any expert
    l[1, :] = -INF
    l[1, 37] = 0.25                                 # one
    l[2, ::2] = -INF
    l[3] = torch.finfo(torch.float32).min           # the lowest number is a number
    l[4, 5] = torch.finfo(torch.float32).min
    l[5, 10:] = -INF
    for bias in (None, torch.zeros(100)):
        if bias is not None:
            bias[[3, 50, 99]] = -INF
            l[6, 3], l[6, 50], l[7, 99] = float("nan"), INF, float("nan")     # out: whatever the logit holds
        ids, w = X.route(l.cuda(), rule_of(X, 12, score, renormalize=renormalize), bias=None if bias is None else bias.cuda())
        ids, w = ids.cpu(), w.cpu().double()
        clean = l if bias is None else torch.where(bias == -INF, torch.full_like(l, -INF), l)
        if bias is None or score == "sigmoid":
            want = R.choose(clean, score, None if bias is None else torch.zeros(100), 12, 1, 1, False)
            if bias is None:
                assert torch.equal(ids, want)
        assert (ids[0] == -1).all() and (w[0] == 0).all()
        assert ids[1].tolist() == [37] + [-1] * 11 and (ids[2] % 2 == 1).all()
        assert (ids[5, :10] >= 0).sum() == (10 if bias is None else 9)
        if bias is not None:
            assert not any((ids == e).any() for e in (3, 50, 99))
        assert ((ids < 0) == (w == 0))[[0, 1, 2, 5, 6, 7]].all()
        ref = R.chosen_weights(clean, score, None, ids, renormalize, 1.0)
        assert torch.isfinite(w).all()
        assert ((w - ref).abs() <= weight_bound(100) * ref + 1e-45).all()
        d = X.route_backward(l.cuda(), rule_of(X, 12, score, renormalize=renormalize), ids.cuda(), torch.ones(8, 12).cuda(),
                             bias=None if bias is None else bias.cuda()).cpu()
        assert torch.isfinite(d).all() and (d[clean == -INF] == 0).all()


def test_what_is_not_a_number_shows(X):
    l = logits_of(4, 70, 9)
    l[1, 66] = float("nan")
    l[2, 3] = INF
    for score in ("softmax", "sigmoid"):
        ids, w = X.route(l.cuda(), rule_of(X, 5, score))
        ids, w = ids.cpu(), w.cpu()
        assert ((ids >= 0) & (ids < 70)).all() and torch.isfinite(w[[0, 3]]).all()
        assert torch.isnan(w[1]).all()
        assert ids[2, 0] == 3 and (torch.isnan(w[2]).all() if score == "softmax" else torch.isfinite(w[2]).all())
        d = X.route_backward(l.cuda(), rule_of(X, 5, score), ids.cuda(), torch.ones(4, 5).cuda()).cpu()
        assert torch.isfinite(d[[0, 3]]).all() and torch.isnan(d[1]).all()


def test_strides_streams_and_no_rows(X):
    wide = logits_of(20, 300, 1).cuda()
    part = wide[3:17:2, 11:111]                      # rows 600 apart, not aligned
    rule = rule_of(X, 7, "softmax")
    ids, w = X.route(part, rule)
    a, b = X.route(part.contiguous(), rule)
    assert torch.equal(ids, a) and torch.equal(w, b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c, d = X.route(part, rule)
    s.synchronize()
    assert torch.equal(ids, c) and torch.equal(w, d)
    ids, w = X.route(wide[:0], rule)
    assert ids.shape == (0, 7) and w.shape == (0, 7)
    assert X.route_backward(wide[:0], rule, ids, w).shape == (0, 300)
    assert X.plan(ids, 300).offsets.tolist() == [0] * 301


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("T,E,k", [(1, 8, 1), (5, 64, 6), (7, 130, 8), (3, 1000, 64), (70, 17, 3)])
def test_gradient_is_the_formulas(X, T, E, k, score, renormalize):
    g = torch.Generator().manual_seed(k)
    for dtype, rest in ((torch.float32, 0.0), (torch.bfloat16, 2.0 ** -8), (torch.float16, 2.0 ** -11)):
        l = (torch.randn(T, E, generator=g) * 1.5).to(dtype)
        l[0, 0] = -INF if E > k else 0.0
        rule = rule_of(X, k, score, renormalize=renormalize, scale=1.7)
        ids, _ = X.route(l.cuda(), rule)
        ids[T - 1, k - 1] = -1                       # a slot that was given up
        dw = torch.randn(T, k, generator=g)
        got = X.route_backward(l.cuda(), rule, ids, dw.cuda()).cpu().double()
        leaf = l.double().requires_grad_(True)
        w = R.chosen_weights(leaf, score, None, ids.cpu(), renormalize, 1.7)
        (want,) = torch.autograd.grad((w * dw.double()).sum(), leaf)
        want = torch.nan_to_num(want)
        # every term of dl_e is at most scale * max |dw|, times s_e (1 for sigmoid); k + 8 roundings beside the score's own
        s = R.scores(l, score, None) if score == "softmax" and not renormalize else torch.ones(T, E, dtype=torch.float64)
        bound = (weight_bound(E) + (k + 8) * 2 * R.U) * 2 * 1.7 * dw.abs().sum(1, keepdim=True).double() * s
        if score == "sigmoid" and renormalize:        # divided by the sum of the chosen, which may be small
            total = (torch.gather(torch.sigmoid(l.double()), 1, ids.cpu().clamp_min(0).long()) * (ids.cpu() >= 0)).sum(1, keepdim=True)
            bound = bound / total.clamp_max(1.0)
        assert ((got - want).abs() <= bound + rest * want.abs() + 1e-7 * (rest > 0)).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
def test_gradient_is_that_of_differences(X, score, renormalize):
    """Central differences of the routed weights themselves, logits far enough apart that the choice stays."""
    g = torch.Generator().manual_seed(3)
    E, k, h = 40, 5, 1.0 / 64
    l = (torch.randperm(E, generator=g).float() / 8 - 2.5)[None]
    dw = torch.randn(1, k, generator=g)
    rule = rule_of(X, k, score, renormalize=renormalize, scale=2.0)
    ids, _ = X.route(l.cuda(), rule)
    got = X.route_backward(l.cuda(), rule, ids, dw.cuda()).cpu().double()[0]
    steps = torch.cat([l + h * torch.eye(E), l - h * torch.eye(E)])
    ids2, w = X.route(steps.cuda(), rule)
    assert (ids2 == ids).all()
    f = (w.cpu().double() * dw.double()).sum(1)
    # third derivatives of a score are below 1; two weights with a few roundings each over 2 h
    bound = 2.0 * dw.abs().sum().item() * (h * h / 6 * 2 + 40 * R.U / h)
    assert ((f[:E] - f[E:]) / (2 * h) - got).abs().max().item() <= bound


@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 6, 64), (9, 7, 3), (64, 1, 5), (65, 1, 5), (300, 4, 100), (2048, 8, 256), (2049, 8, 1024),
                                   (70000, 1, 1000), (9000, 4, 7)])
def test_order_is_stable_and_whole(X, T, k, E):
    g = torch.Generator().manual_seed(T)
    ids = torch.randint(-2, E + 2, (T, k), generator=g).int()
    if E > 3:
        ids[ids == 2] = 3                            # one expert without rows, one with many
    p = X.plan(ids.cuda(), E)
    offsets, blks, slots, places = R.order_of(ids, E)
    assert p.offsets.tolist() == offsets and p.blocks.tolist() == blks
    assert p.slots.tolist() == slots and p.places.tolist() == places
    assert blks[-1] <= p.max_blocks()


def test_order_of_nothing_and_of_one_expert(X):
    p = X.plan(torch.full((50, 3), -1, dtype=torch.int32).cuda(), 9)
    assert p.offsets.tolist() == [0] * 10 and (p.slots == -1).all() and (p.places == -1).all()
    p = X.plan(torch.full((700, 3), 8, dtype=torch.int32).cuda(), 9)
    assert p.offsets.tolist() == [0] * 9 + [2100] and p.slots.tolist() == list(range(2100))


def test_same_bits_every_time(X):
    l = torch.randn(3000, 200, generator=torch.Generator().manual_seed(1)).cuda()
    rule = rule_of(X, 8, "softmax", renormalize=False)
    a = X.route(l, rule)
    pa = X.plan(a[0], 200)
    for _ in range(3):
        b = X.route(l, rule)
        pb = X.plan(b[0], 200)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(pa.slots, pb.slots)


def test_learned_centroids_route_to_the_nearest(X):
    """With the scores x.c and the bias -|c|^2 / 2 on them as logits the best expert is the nearest centroid."""
    g = torch.Generator().manual_seed(4)
    x, c = torch.randn(500, 24, generator=g), torch.randn(37, 24, generator=g)
    score = x @ c.t() - 0.5 * (c * c).sum(1)
    ids, _ = X.route(score.cuda(), rule_of(X, 2, "softmax"))
    near = torch.cdist(x.double(), c.double()).topk(2, largest=False).indices
    assert (ids.cpu().long() == near).float().mean() > 0.999
    assert math.isclose(float((ids.cpu()[:, 0].long() == near[:, 0]).float().mean()), 1.0, abs_tol=0.002)
