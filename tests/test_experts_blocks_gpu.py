"""Products in 8-bit blocks on the GPU: bringing to 8 bits bit for bit, products and gradients against 64 bits."""
import pytest
import torch

from tests import experts_rules as R

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ROUNDING = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; there is no CPU fallback")
    from paper_1505_04956_amd import experts
    return experts


def data(rows, cols, seed, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(cols, generator=g))
    if rows > 2 and cols > 130:
        x[1, :128] = 0.0                                # a block of zeros
        x[2] *= 1e-4
    return x.to(dtype)


def same_bits(got, want):
    return torch.equal(got.cpu().view(torch.uint8), want.contiguous().view(torch.uint8))


def same_scales(got, want):
    return torch.equal(torch.nan_to_num(got.cpu(), nan=-1.0), torch.nan_to_num(want, nan=-1.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 127), (5, 129), (130, 257), (64, 1000), (257, 64), (300, 8)])
def test_to_eight_bits(X, rows, cols, dtype):
    x = data(rows, cols, rows + cols, dtype)
    q, s = R.to_blocks(x.float())
    got = X.quantize(x.cuda())
    assert same_bits(got.values, q.view(rows, -1)) and same_scales(got.scales, s)
    q, s = R.to_blocks(x.float().t())
    got = X.quantize(x.cuda(), turned=True)
    assert same_bits(got.values, q.view(cols, -1)) and same_scales(got.scales, s)
    q, s = R.to_squares(x.float())
    got = X.quantize_weights(x.cuda())
    assert same_bits(got.values, q) and same_scales(got.scales, s)
    q, s = R.to_squares(x.float().t())
    got = X.quantize_weights(x.cuda(), turned=True)
    assert same_bits(got.values, q) and same_scales(got.scales, s)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (5, 129), (128, 64), (130, 257), (257, 200)])
def test_both_ways_at_once(X, rows, cols, dtype):
    """What a training step takes of a matrix: the rows' and the transpose's blocks, as they are one by one."""
    base = data(rows, cols + 24, rows, dtype).cuda()
    for x in (base[:, :cols], base[:, :cols].contiguous()):
        a, b = X._quantized_both(x)
        for got, want in ((a, X.quantize(x)), (b, X.quantize(x, turned=True))):
            n = want.values.numel()
            assert torch.equal(got.memory[:n], want.values.view(torch.uint8).reshape(-1))
            assert torch.equal(got.memory[n:].view(torch.float32), want.scales.reshape(-1))


def test_turned_squares_are_the_same_numbers(X):
    w = data(3 * 200, 300, 2).view(3, 200, 300)
    a, b = X.quantize_weights(w.cuda()), X.quantize_weights(w.cuda(), turned=True)
    assert torch.equal(a.scales, b.scales.transpose(1, 2))
    assert torch.equal(a.values[:, :, :300].view(torch.uint8), b.values[:, :, :200].view(torch.uint8).transpose(1, 2))
    one = X.quantize_weights(w[1].contiguous().cuda())
    assert torch.equal(one.values.view(torch.uint8), a.values[1].view(torch.uint8)) and torch.equal(one.scales, a.scales[1])


@pytest.mark.parametrize("dtype", TYPES)
def test_to_eight_bits_of_strided_rows(X, dtype):
    base = data(40, 700, 3, dtype).cuda()
    for x in (base[::3, 5:400], base[1:20, 8:136], base[:1, 3:], base[:, 640:]):
        for turned in (False, True):
            a, b = X.quantize(x, turned=turned), X.quantize(x.contiguous(), turned=turned)
            assert torch.equal(a.values.view(torch.uint8), b.values.view(torch.uint8)) and torch.equal(a.scales, b.scales)


def test_extremes_of_a_block(X):
    x = torch.zeros(8, 256)
    x[0, 3], x[0, 200] = 3.3e38, 1e-45                  # the largest numbers, and the smallest
    x[1, :4] = torch.tensor([1e-31, -1e-33, 1e-30, 0.0])
    x[2, :3] = torch.tensor([448.0, 17.0, 0.0009765625])     # a tie between two e4m3 numbers, and half of the smallest
    x[3, 7] = float("inf")
    x[4, 130] = float("nan")
    x[5, :128] = -1.0
    x[6, 255] = -0.0
    q, s = R.to_blocks(x)
    got = X.quantize(x.cuda())
    assert same_scales(got.scales, s)
    ok = torch.isfinite(s.t())
    v = got.values.cpu().view(8, 2, 128)
    assert torch.equal(v[ok].view(torch.uint8), q[ok].view(torch.uint8))
    assert torch.isnan(s[0, 3]) and torch.isnan(s[1, 4]) and ok.sum() == 14
    # a block that is not all numbers spoils its own row of a product, and nothing else
    w = X.quantize_weights(data(130, 256, 1).cuda())
    for exact in (False, True):
        y = X.product(got, w, torch.float32, exact=exact)
        assert torch.isnan(y[[3, 4]]).all() and torch.isfinite(y[[1, 2, 5, 6, 7]]).all()
    y = X.linear(x.cuda(), w)                           # few rows: brought to 8 bits inside the product
    assert torch.isnan(y[[3, 4]]).all() and torch.isfinite(y[[1, 2, 5, 6, 7]]).all()


def bounds(a, b, exact, dtype, want):
    """|a| |b| summed, times: 128 products a block in 32 bits (the 16-bit instruction: 4 sums of 32, each within 6 half-ulps as the
    matrix cores add) or the 8-bit instruction's 7 * 2^-14 of the largest of eight; then a scale product, a fma and an addition a block."""
    m = a.abs() @ b.abs().t()
    kb = -(-a.shape[1] // 128)
    per = (4 * 6 + 4 + kb) * 2 * R.U + (0.0 if exact else 7 * 2.0 ** -14)
    return m * per + ROUNDING[dtype] * want.abs() + (6e-8 if dtype == torch.float16 else 1e-38)


SIZES = [(1, 1, 1), (1, 64, 100), (3, 5, 129), (16, 257, 128), (17, 100, 1000), (33, 130, 384), (64, 64, 64), (127, 129, 500), (128, 128, 128),
         (129, 1, 257), (200, 300, 300), (300, 260, 1100), (1, 1001, 2049), (520, 20, 130)]


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("rows,outs,cols", SIZES)
def test_product(X, rows, outs, cols, exact):
    for n, dtype in enumerate(TYPES):
        x, w = data(rows, cols, n + 1), data(outs, cols, n + 7)
        a, b, c = X.quantize(x.cuda()), X.quantize_weights(w.cuda()), X.quantize(w.cuda())
        A, Bq, Cq = R.rounded(x), R.from_squares(*R.to_squares(w))[:, :cols], R.rounded(w)
        for other, O in ((b, Bq), (c, Cq)):
            y = X.product(a, other, dtype, exact=exact).cpu().double()
            want = A @ O.t()
            assert ((y - want).abs() <= bounds(A, O, exact, dtype, want)).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 2, 9, 16])
@pytest.mark.parametrize("outs,cols", [(1, 1), (100, 77), (257, 128), (64, 1000), (300, 2056), (48, 96)])
def test_few_rows(X, rows, outs, cols, dtype):
    """Rows that the product brings to 8 bits itself."""
    x, w = data(rows, cols, rows, dtype), data(outs, cols, 3)
    A, Bq = R.rounded(x.float()), R.from_squares(*R.to_squares(w))[:, :cols]
    b, want = X.quantize_weights(w.cuda()), R.rounded(x.float()) @ Bq.t()
    for y in (X.linear(x.cuda(), b), X.linear(torch.cat([x, x], 1).cuda()[:, :cols], b)):
        assert y.dtype == dtype
        assert ((y.cpu().double() - want).abs() <= bounds(A, Bq, dtype == torch.float32, dtype, want)).all()


def test_products_say_the_same_however_many_rows(X):
    """A row's result does not depend on its neighbours or on how many there are, but for the order in which blocks are added."""
    w = X.quantize_weights(data(200, 640, 4).cuda())
    x = data(300, 640, 5).cuda()
    whole = X.linear(x, w)
    for n in (1, 16, 17, 128, 129):
        part = X.linear(x[100:100 + n], w)
        assert ((part - whole[100:100 + n]).abs() <= 1e-5 * whole.abs().max()).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,outs,cols", [(1, 1, 1), (5, 130, 77), (128, 128, 128), (200, 300, 150), (300, 65, 513)])
def test_gradients_are_the_formulas(X, rows, outs, cols, dtype):
    x, w, d = data(rows, cols, 1, dtype), data(outs, cols, 2), data(rows, outs, 3, dtype)
    y, kept = X.linear(x.cuda(), X.quantize_weights(w.cuda()), train=True)
    d_x, d_w = X.linear_backward(d.cuda(), kept, X.quantize_weights(w.cuda(), turned=True))
    Wq = R.from_squares(*R.to_squares(w))[:, :cols]
    D = R.rounded(d.float())
    want = D @ Wq
    assert d_x.dtype == dtype and ((d_x.cpu().double() - want).abs() <= bounds(D, Wq.t().contiguous(), dtype == torch.float32, dtype, want)).all()
    Dt, Xt = R.rounded(d.float().t()), R.rounded(x.float().t())
    want = Dt @ Xt.t()
    assert d_w.dtype == torch.float32 and ((d_w.cpu().double() - want).abs() <= bounds(Dt, Xt, True, torch.float32, want)).all()


def whole_numbers(rows, cols, seed, low=-3, high=3):
    """Small whole numbers with a 448 in each block along both ways, so that every scale is one and 8 bits hold all of it."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randint(low, high + 1, (rows, cols), generator=g).float()
    x[::128] = 448.0
    x[:, ::128] = 448.0
    return x


def test_gradients_are_those_of_differences(X):
    """Where 8 bits hold everything the layer is linear, and differences are exact: steps of one in x and in w."""
    rows, outs, cols = 130, 140, 150
    x, w = whole_numbers(rows, cols, 1), whole_numbers(outs, cols, 2)
    d = whole_numbers(rows, outs, 3)
    f = lambda x, w: (X.linear(x.cuda(), X.quantize_weights(w.cuda())).double() * d.cuda().double()).sum().item()  # noqa: E731
    _, kept = X.linear(x.cuda(), X.quantize_weights(w.cuda()), train=True)
    d_x, d_w = X.linear_backward(d.cuda(), kept, X.quantize_weights(w.cuda(), turned=True))
    for i, j in ((1, 1), (129, 149), (64, 130), (127, 5)):
        up, down = x.clone(), x.clone()
        up[i, j] += 1
        down[i, j] -= 1
        assert (f(up, w) - f(down, w)) / 2 == d_x[i, j].item()
    for i, j in ((1, 1), (139, 149), (100, 130), (127, 5)):
        up, down = w.clone(), w.clone()
        up[i, j] += 1
        down[i, j] -= 1
        assert (f(x, up) - f(x, down)) / 2 == d_w[i, j].item()


def test_no_rows(X):
    w = X.quantize_weights(data(70, 90, 1).cuda())
    y, kept = X.linear(torch.empty(0, 90, device="cuda"), w, train=True)
    assert y.shape == (0, 70)
    d_x, d_w = X.linear_backward(torch.empty(0, 70, device="cuda"), kept, X.quantize_weights(data(70, 90, 1).cuda(), turned=True))
    assert d_x.shape == (0, 90) and d_w.shape == (70, 90) and (d_w == 0).all()


def test_offsets_beyond_32_bits(X):
    """Rows far down a matrix of more than 2^32 bytes."""
    rows, cols = 300_000, 8192
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("needs 24 GB")
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    at = [0, 131_072, 262_144, 299_999]
    x[at] = data(4, cols, 8).to(torch.bfloat16).cuda()
    q = X.quantize(x)
    few = X.quantize(x[at + list(range(1, 200))])                      # (enough rows for the same kernel: the same bits)
    assert torch.equal(q.values[at].view(torch.uint8), few.values[:4].view(torch.uint8)) and torch.equal(q.scales[:, at], few.scales[:, :4])
    w = X.quantize_weights(data(40, cols, 9).cuda())
    y = X.product(q, w, torch.float32)
    assert torch.equal(y[at], X.product(few, w, torch.float32)[:4]) and int((y.abs().sum(1) > 0).sum()) == 4


def test_in_a_graph(X):
    """Captured once, replayed with other inputs, other work in between."""
    w = X.quantize_weights(data(300, 640, 4).cuda())
    for rows in (1, 40):
        x = data(rows, 640, 5).cuda()
        X.linear(x, w)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = X.linear(x, w)
        for seed in (6, 7, 8):
            x.copy_(data(rows, 640, seed))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, X.linear(x.clone(), w))
