"""4-bit floating point on the GPU: bringing to 4 bits bit for bit, products and experts against 64 bits."""
import pytest
import torch

from tests import experts_rules as R
from tests import micro_rules as Q

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ROUNDING = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SMALLEST = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 6e-8}


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; there is no CPU fallback")
    from paper_1505_04956_amd import micro
    return micro


@pytest.fixture(scope="module")
def X(M):
    from paper_1505_04956_amd import experts
    return experts


def data(rows, cols, seed, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(cols, generator=g))
    if rows > 2 and cols > 70:
        x[1, :64] = 0.0
        x[2] *= 1e-4
    return x.to(dtype)


def same(m, x):
    code, s = Q.to_four(x.float())
    return torch.equal(m.scales.cpu().long(), s) and torch.equal(m.values.cpu(), Q.packed(code))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 31), (5, 33), (130, 257), (64, 1000), (257, 64), (300, 8), (2, 256), (7, 255)])
def test_to_four_bits_and_back(M, rows, cols, dtype):
    x = data(rows, cols, rows + cols, dtype)
    m = M.quantize(x.cuda())
    assert (m.rows, m.cols, m.count) == (rows, cols, 1) and same(m, x)
    for back in TYPES:
        got = M.expand(m, back)
        assert got.dtype == back and torch.equal(got.cpu(), Q.matrix_of(m).to(back))


@pytest.mark.parametrize("dtype", TYPES)
def test_strided_rows_and_experts(M, dtype):
    base = data(40, 700, 3, dtype).cuda()
    for x in (base[::3, 5:400], base[1:20, 8:136], base[:1, 3:], base[:, 640:]):
        a, b = M.quantize(x), M.quantize(x.contiguous())
        assert torch.equal(a.values, b.values) and torch.equal(a.scales, b.scales)
    w = data(6 * 5, 300, 4, dtype).view(6, 5, 300).cuda()
    m = M.quantize(w)
    assert m.count == 6 and m.rows == 5 and M.expand(m).shape == (6, 5, 300)
    for e in range(6):
        one = M.quantize(w[e])
        assert torch.equal(one.values, m.values[e]) and torch.equal(one.scales, m.scales[e])
    assert torch.equal(M.expand(m)[3].cpu().double(), Q.matrix_of(m)[3])


def test_one_expert_of_many(M):
    """Its scales begin at a multiple of eight bytes."""
    m = M.quantize(data(5 * 33, 700, 1).view(5, 33, 700).cuda())
    x = data(40, 700, 2).cuda()
    for e in range(5):
        one = M.Micro(m.values[e], m.scales[e], 700)
        assert torch.equal(M.expand(one), M.expand(m)[e])
        for rows in (1, 20, 40):
            want = M.linear(x[:rows], M.Micro(m.values[e].clone(), m.scales[e].clone(), 700))
            assert torch.equal(M.linear(x[:rows], one), want)
        ids = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
        a = M.Micro(m.values[e:e + 1], m.scales[e:e + 1], 700)
        q, v = Q.four(x[:2].cpu()), Q.matrix_of(one)
        close(M.experts(x[:2], ids, torch.ones(2, 1, device="cuda"), a), q @ v.t(), Q.product_bound(q.abs() @ v.abs().t(), 700), torch.float32)


def test_extremes_of_a_block(M):
    x = torch.zeros(14, 300)
    x[0, 3], x[0, 200] = 3.4028234e38, 1.5e-45                      # the largest number, and nearly the smallest
    x[1, :4] = torch.tensor([1e-37, -1e-38, 6e-39, 3e-39])          # near the smallest scale
    x[2, :9] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25])      # ties
    x[3, :2] = torch.tensor([6.9999995, 1.0])                       # cut at 6
    x[4, :2] = torch.tensor([7.0, 1.0])                             # the next scale
    x[5, 7] = float("inf")
    x[6, 40] = float("nan")
    x[7, 299] = -float("inf")
    x[8, :32] = -1.0
    x[9, 31] = -0.0
    x[10, 0] = 2.0 ** -126
    x[11, 0] = 2.0 ** -149
    x[12, :2] = torch.tensor([1.9999999, 1.75])
    x[13, :2] = torch.tensor([1.7499999, -1.5])
    m = M.quantize(x.cuda())
    code, s = Q.to_four(x)
    assert torch.equal(m.scales.cpu().long(), s)
    fine = (s != 255).repeat_interleave(32, 1)
    assert torch.equal(Q.codes(m.values)[fine], code[fine]) and (s == 255).sum() == 3
    # a block that is not all numbers spoils its own row of a product, and nothing else
    w = M.quantize(data(130, 300, 1).cuda())
    for y in (M.product(m, w, torch.float32), M.linear(x.cuda(), w)):
        assert torch.isnan(y[[5, 6, 7]]).all() and torch.isfinite(y[1:5]).all() and torch.isfinite(y[8:]).all()
    y = M.product(w, m, torch.float32)
    assert torch.isnan(y[:, [5, 6, 7]]).all() and torch.isfinite(y[:, 1:5]).all()
    # rows in 32 or 64 places of tiles
    many = torch.cat([x] * 20)
    y = M.linear(many.cuda(), w).view(20, 14, 130)
    assert torch.isnan(y[:, [5, 6, 7]]).all() and torch.isfinite(y[:, 1:5]).all()


SIZES = [(1, 1, 1), (1, 64, 100), (3, 5, 129), (16, 257, 128), (17, 100, 1000), (32, 33, 513), (33, 130, 384), (64, 64, 64), (127, 129, 500), (128, 128, 256),
         (129, 257, 257), (200, 1000, 300), (300, 40, 2049), (513, 700, 96), (2, 20, 5000)]


def close(got, want, bound, dtype):
    off = (got.cpu().double() - want).abs()
    allowed = bound + ROUNDING[dtype] * (want.abs() + bound) + SMALLEST[dtype]
    assert (off <= allowed).all(), float((off / allowed).max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,outs,cols", SIZES)
def test_products(M, rows, outs, cols, dtype):
    x, w = data(rows, cols, rows, dtype), data(outs, cols, outs + 1) * 0.1
    mw = M.quantize(w.cuda())
    a, b = Q.four(x.float()), Q.four(w)
    want, bound = a @ b.t(), Q.product_bound(a.abs() @ b.abs().t(), cols)
    close(M.linear(x.cuda(), mw), want, bound, dtype)
    close(M.product(M.quantize(x.cuda()), mw, dtype), want, bound, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tile,rows,outs,cols", [(64, 300, 500, 2100), (64, 1000, 700, 900), (128, 2048, 2048, 300), (128, 1100, 4000, 70), (128, 2000, 2000, 1500), (64, 4100, 1030, 2049), (128, 4000, 1020, 2049),
                                                 (256, 4096, 4096, 1100), (256, 3900, 4090, 2049), (256, 8100, 2040, 1300)])
def test_large_tiles(M, tile, rows, outs, cols, dtype):
    from paper_1505_04956_amd import binding as B
    x, w = data(rows, cols, 5, dtype), data(outs, cols, 6)
    ma, mw = M.quantize(x.cuda()), M.quantize(w.cuda())
    assert B.asgd_block_product_form(ma._c, mw._c, B.PRODUCT_ALL, 0, None) == {64: B.PRODUCT_FORM_TILES_64, 128: B.PRODUCT_FORM_TILES_128, 256: B.PRODUCT_FORM_TILES_256}[tile]
    y = M.product(ma, mw, dtype)
    pick = torch.cat([torch.arange(0, rows, 97), torch.arange(rows - 300, rows)])
    a, b = Q.four(x[pick].float()), Q.four(w)
    close(y[pick.cuda()], a @ b.t(), Q.product_bound(a.abs() @ b.abs().t(), cols), dtype)


def test_scales_far_apart(M):
    """Blocks whose scales are far apart, products that cancel: what is dropped is small beside the magnitudes that were added."""
    g = torch.Generator().manual_seed(2)
    x = torch.randn(40, 1024, generator=g) * torch.exp2(torch.randint(-30, 30, (40, 32), generator=g).float()).repeat_interleave(32, 1)
    w = torch.randn(50, 1024, generator=g) * torch.exp2(torch.randint(-30, 30, (50, 32), generator=g).float()).repeat_interleave(32, 1)
    x[:, 512:], w[:, 512:] = x[:, :512], -w[:, :512]
    a, b = Q.four(x), Q.four(w)
    want, bound = a @ b.t(), Q.product_bound(a.abs() @ b.abs().t(), 1024)
    mw = M.quantize(w.cuda())
    close(M.linear(x.cuda(), mw), want, bound, torch.float32)
    close(M.linear(x[:7].cuda(), mw), want[:7], bound[:7], torch.float32)


def test_nothing_to_do(M):
    w = M.quantize(data(20, 300, 1).cuda())
    assert M.linear(torch.empty(0, 300, device="cuda"), w).shape == (0, 20)
    assert M.quantize(torch.empty(0, 300, device="cuda")).values.shape == (0, 256)
    assert M.expand(M.quantize(torch.empty(0, 300, device="cuda"))).shape == (0, 300)
    w = M.quantize(data(60, 300, 1).view(3, 20, 300).cuda())
    ids, weights = torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, device="cuda")
    assert M.experts(torch.empty(0, 300, device="cuda"), ids, weights, w).shape == (0, 20)
    for T in (1, 16, 40):
        ids = torch.full((T, 2), -1, dtype=torch.int32, device="cuda")
        y = M.experts(data(T, 300, 2).cuda(), ids, torch.ones(T, 2, device="cuda"), w)
        assert torch.equal(y, torch.zeros(T, 20, device="cuda"))


def routed(T, E, k, seed, padding=0.1):
    g = torch.Generator().manual_seed(seed)
    ids = torch.argsort(torch.randn(T, E, generator=g) + torch.randn(E, generator=g), dim=1)[:, :k].int().contiguous()
    weights = torch.rand(T, k, generator=g)
    out = torch.rand(T, generator=g) < padding
    ids[out] = -1
    ids[torch.rand(T, k, generator=g) < padding / 2] = E + 3
    return ids, weights


def experts_64(x, ids, weights, w):
    """(result, bound) of experts in 4 bits; w [E, N, K] float32."""
    q, T, N = Q.four(x.float()), x.shape[0], w.shape[1]
    y, off = torch.zeros(T, N, dtype=torch.float64), torch.zeros(T, N, dtype=torch.float64)
    for e in range(w.shape[0]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if len(t):
            b, c = Q.four(w[e]), weights[t, j].double()[:, None]
            y.index_add_(0, t, c * (q[t] @ b.t()))
            m = q[t].abs() @ b.abs().t()
            off.index_add_(0, t, c.abs() * (Q.product_bound(m, x.shape[1]) + 2 * (ids.shape[1] + 2) * Q.U * m))
    return y, off


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k,N,K", [(1, 8, 2, 40, 300), (1, 64, 6, 130, 513), (16, 5, 3, 17, 64), (17, 9, 2, 100, 257), (24, 100, 5, 100, 500), (300, 7, 2, 129, 260),
                                       (700, 3, 1, 256, 1000), (200, 300, 4, 20, 70),
                                       (200, 300, 4, 200, 70), (1500, 120, 2, 300, 60), (1200, 40, 1, 300, 260), (900, 50, 1, 300, 600), (3000, 500, 4, 100, 70), (1000, 100, 1, 300, 200),
                                       (1100, 3, 2, 300, 1300), (2100, 5, 1, 129, 2600), (40, 6, 2, 17, 8300)])
def test_experts(M, T, E, k, N, K, dtype):
    x, w = data(T, K, T, dtype), (data(E * N, K, E) * 0.1).view(E, N, K)
    ids, weights = routed(T, E, k, T + E)
    want, bound = experts_64(x, ids, weights, w)
    got = M.experts(x.cuda(), ids.cuda(), weights.cuda(), M.quantize(w.cuda()))
    close(got, want, bound, dtype)


def test_the_same_expert_twice(M):
    x, w = data(5, 300, 1), data(3 * 20, 300, 2).view(3, 20, 300)
    ids = torch.tensor([[1, 1, 1], [2, 0, 2], [0, 0, 1], [-1, 2, 2], [5, 5, 5]], dtype=torch.int32)
    weights = torch.rand(5, 3)
    want, bound = experts_64(x, ids, weights, w)
    mw = M.quantize(w.cuda())
    close(M.experts(x.cuda(), ids.cuda(), weights.cuda(), mw), want, bound, torch.float32)
    close(M.experts(x.repeat(8, 1).cuda(), ids.repeat(8, 1).cuda(), weights.repeat(8, 1).cuda(), mw), want.repeat(8, 1), bound.repeat(8, 1), torch.float32)


@pytest.mark.parametrize("T,k,E,N", [(9, 2, 5, 40), (300, 2, 3, 40), (300, 2, 3, 200), (600, 2, 100, 400), (600, 2, 50, 400)])
def test_products_by_place(M, X, T, k, E, N):
    """gather and places, and places that are not in use left as they were."""
    ids, _ = routed(T, E, k, 3)
    x, w = data(T, 300, 1), data(E * N, 300, 2).view(E, N, 300)
    order, mw = X.plan(ids.cuda(), E), M.quantize(w.cuda())
    offsets, _, slots, _ = R.order_of(ids, E)
    used = offsets[-1]
    token = torch.tensor(slots[:used]) // k
    expert = torch.tensor([e for e in range(E) for _ in range(offsets[e + 1] - offsets[e])])
    q = Q.four(x)
    want = torch.stack([Q.four(w[e]) @ q[t] for e, t in zip(expert.tolist(), token.tolist())])
    bound = torch.stack([Q.product_bound(Q.four(w[e]).abs() @ q[t].abs(), 300) for e, t in zip(expert.tolist(), token.tolist())])
    a = M.quantize(x.cuda())
    close(M.product(a, mw, torch.float32, order, gather=True)[:used], want, bound, torch.float32)
    rows = torch.zeros(T * k, 300)
    rows[:used] = x[token]
    close(M.product(M.quantize(rows.cuda()), mw, torch.float32, order)[:used], want, bound, torch.float32)
    from paper_1505_04956_amd import binding as B
    out = torch.full((T * k, N), 7.0, device="cuda")
    B.asgd_block_product(a._c, mw._c, B.PRODUCT_GATHER, 0, order._c, out.data_ptr(), B.TYPE_F32, N, torch.cuda.current_stream().cuda_stream)
    assert (out[used:] == 7.0).all() and used < T * k
    close(out[:used], want, bound, torch.float32)


def test_results_apart(M):
    """Rows of the result further apart than they are long, at an odd address: what lies between them is left alone."""
    from paper_1505_04956_amd import binding as B
    for rows in (5, 40, 300):
        x, w = data(rows, 300, 1, torch.bfloat16), data(50, 300, 2)
        ma, mw = M.quantize(x.cuda()), M.quantize(w.cuda())
        want = M.product(ma, mw, torch.bfloat16)
        out = torch.full((rows * 61 + 9,), 7.0, device="cuda", dtype=torch.bfloat16)
        B.asgd_block_product(ma._c, mw._c, B.PRODUCT_ALL, 0, None, out.data_ptr() + 2 * 3, B.TYPE_BF16, 61, torch.cuda.current_stream().cuda_stream)
        got = out[3:3 + rows * 61].view(rows, 61)
        assert torch.equal(got[:, :50], want) and (got[:, 50:] == 7.0).all() and (out[:3] == 7.0).all() and (out[-6:] == 7.0).all()
        e = torch.full((rows * 301 + 1,), 7.0, device="cuda", dtype=torch.bfloat16)
        B.asgd_block_expand(ma._c, e.data_ptr() + 2, B.TYPE_BF16, 301, torch.cuda.current_stream().cuda_stream)
        got = e[1:].view(rows, 301)
        assert torch.equal(got[:, :300], M.expand(ma, torch.bfloat16)) and (got[:, 300] == 7.0).all()


def test_the_same_bits_again_on_a_stream_and_in_a_graph(M):
    x, w = data(24, 500, 1, torch.bfloat16).cuda(), M.quantize(data(9 * 70, 500, 2).view(9, 70, 500).cuda())
    one = M.quantize(data(70, 500, 3).cuda())
    ids, weights = (t.cuda() for t in routed(24, 9, 3, 1))
    def calls():
        return (M.experts(x, ids, weights, w), M.experts(x[:5], ids[:5], weights[:5], w), M.linear(x, one), M.linear(x[:2], one), M.expand(M.quantize(x)))
    want = [t.clone() for t in calls()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = calls()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls()
    for n in range(3):
        for t in held:
            t.zero_()
        x.copy_(data(24, 500, 1 + n, torch.bfloat16))
        want = [t.clone() for t in calls()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_beyond_four_gigabytes(M, X):
    """Weights, rows and results whose places pass 32 bits: what lies at their ends is found."""
    from paper_1505_04956_amd import layer as L
    E, N, K = 520, 2048, 8192                                       # 4.4 GB of values
    w = data(N, K, 1) * 0.1
    one = M.quantize(w.cuda())
    values = torch.zeros(E, N, K // 2, dtype=torch.uint8, device="cuda")
    scales = torch.full((E, N, K // 32), 127, dtype=torch.uint8, device="cuda")
    values[-1], scales[-1] = one.values, one.scales
    many = M.Micro(values, scales, K)
    b = Q.four(w)
    for T in (1, 40):
        x = data(T, K, T, torch.bfloat16)
        a = Q.four(x.float())
        want, bound = a @ b.t(), Q.product_bound(a.abs() @ b.abs().t(), K)
        ids = torch.full((T, 1), E - 1, dtype=torch.int32, device="cuda")
        close(M.experts(x.cuda(), ids, torch.ones(T, 1, device="cuda"), many), want, bound + 8 * Q.U * want.abs(), torch.bfloat16)
        order = X.plan(ids, E)
        close(M.product(M.quantize(x.cuda()), many, torch.float32, order, gather=True), want, bound, torch.float32)
    # a layer whose second matrix this is: h is 8192 columns
    H, D = K, 64
    up = data(2 * H, D, 5) * 0.1
    u = M.quantize(up.cuda())
    uv, us = torch.zeros(E, 2 * H, 128, dtype=torch.uint8, device="cuda"), torch.full((E, 2 * H, 8), 127, dtype=torch.uint8, device="cuda")
    uv[-1], us[-1] = u.values, u.scales
    x = data(3, D, 9)
    logits = torch.full((3, E), -float("inf"))
    logits[:, -1] = 1.0
    y, ids, weights = L.layer(x.cuda(), logits.cuda(), X.Rule(1), M.Micro(uv, us, D), many)
    assert (ids == E - 1).all() and (weights == 1).all()
    want, bound = Q.layer(x, torch.zeros(3, 1, dtype=torch.int32), torch.ones(3, 1), Q.matrix_of(u)[None], Q.matrix_of(one)[None], 4, False)
    close(y, want, bound, torch.float32)
    del values, scales, many, uv, us
    # rows of activations, and the results of bringing them to 4 bits and back
    rows = (1 << 19) + 130
    v, s = torch.zeros(rows, K // 2, dtype=torch.uint8, device="cuda"), torch.full((rows, K // 32), 127, dtype=torch.uint8, device="cuda")
    assert v.numel() > 1 << 31
    tail = data(70, K, 3)
    t = M.quantize(tail.cuda())
    v[-70:], s[-70:] = t.values, t.scales
    small = M.quantize((data(40, K, 4) * 0.1).cuda())
    q, z = Q.four(tail), Q.matrix_of(small)
    y = M.product(M.Micro(v, s, K), small, torch.float32)
    close(y[-70:], q @ z.t(), Q.product_bound(q.abs() @ z.abs().t(), K), torch.float32)
    assert (y[:-70] == 0).all()
    back = M.expand(M.Micro(v, s, K), torch.bfloat16)               # 8.6 GB
    assert torch.equal(back[-70:].cpu().double(), Q.matrix_of(t).bfloat16().double()) and (back[:1000] == 0).all()
    again = M.quantize(back)
    assert torch.equal(again.values[-70:], t.values)


def test_gathered_scales_beyond_four_gigabytes(M, X):
    """Gathered rows of activations whose scales lie beyond 2^32 bytes of the first: they are their own, not those 2^32 bytes before."""
    K, used = 1 << 20, 6
    T = (1 << 32) // (K // 32) + used
    tail = data(used, K, 1).abs() * 64                              # of one sign: no sum hides a scale that is not its own
    w = data(20, K, 2).abs()
    q, small = M.quantize(tail.cuda()), M.quantize(w.cuda())
    values = torch.empty(T, K // 2, dtype=torch.uint8, device="cuda")   # 69 GB, of which the rows at its ends are written and read
    scales = torch.full((T, K // 32), 127, dtype=torch.uint8, device="cuda")
    assert (T - used) * scales.stride(0) == 1 << 32
    values[-used:], scales[-used:] = q.values, q.scales
    ids = torch.full((T, 1), -1, dtype=torch.int32, device="cuda")
    ids[-used:] = 0
    a, b = Q.four(tail), Q.four(w)
    want = a @ b.t()
    y = M.product(M.Micro(values, scales, K), M.Micro(small.values[None], small.scales[None], K), torch.float32, X.plan(ids, 1), gather=True)
    close(y[:used], want, Q.product_bound(want, K), torch.float32)  # (the places in use are the first)


@pytest.mark.parametrize("rows", [1, 3, 16, 17, 32])
def test_few_rows_of_wide_results(M, rows):
    """Four strips of the weights a workgroup, and more runs than are brought to 4 bits at a time."""
    N, K = 33_000, 17 * 256
    g = torch.Generator(device="cuda").manual_seed(rows)
    values = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(118, 128, (N, K // 32), generator=g, device="cuda", dtype=torch.uint8)
    w, x = M.Micro(values, scales, K), data(rows, K, rows, torch.float16)
    pick = torch.cat([torch.arange(0, N, 331), torch.arange(N - 40, N)])
    a, b = Q.four(x.float()), Q.from_four(Q.codes(values[pick.cuda()]), scales[pick.cuda()].cpu())
    want, bound = a @ b.t(), Q.product_bound(a.abs() @ b.abs().t(), K)
    close(M.product(M.quantize(x.cuda()), w, torch.float32)[:, pick.cuda()], want, bound, torch.float32)
    close(M.linear(x.float().cuda(), w)[:, pick.cuda()], want, bound, torch.float32)


def test_the_largest_numbers(M):
    """From 1.75 * 2^127 on there is no larger scale whose numbers are finite: up to eight times the scale are cut to six, by a quarter at most."""
    top = [1.75 * 2.0 ** 127, 3.4028234663852886e38, 1.7499999 * 2.0 ** 127, 1.5 * 2.0 ** 127, 2.0 ** 127, 1.75 * 2.0 ** 126, 1.7499999 * 2.0 ** 126]
    x = torch.zeros(len(top), 32)
    x[:, 0], x[:, 1] = torch.tensor(top, dtype=torch.float64).float(), -2.0 ** 125
    m = M.quantize(x.cuda())
    assert same(m, x)
    got = M.expand(m).cpu().double()
    assert torch.isfinite(got).all()
    share = (got[:, 0] / x[:, 0].double()).tolist()
    assert share[1] == pytest.approx(0.75, abs=1e-6) and all(0.75 <= v < 6 / 7 + 1e-6 for v in share[:2]) and all(6 / 7 - 1e-6 <= v <= 8 / 7 + 1e-6 for v in share[2:])
    assert (m.scales.cpu()[:5, 0] == 252).all() and got[0, 0] == 6 * 2.0 ** 125
