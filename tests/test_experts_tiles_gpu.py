"""Every kernel that a product can take, with remainders, against 64 bits: what the library would take is asked for, so that another rule
does not leave one of them without a test."""
import ctypes as C

import pytest
import torch

from paper_1505_04956_amd import binding as B
from tests import experts_rules as R
from tests.test_experts_blocks_gpu import ROUNDING, TYPES, data

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a HIP device; there is no CPU fallback")
    from paper_1505_04956_amd import experts
    return experts


def operands(X, rows, outs, cols, squares):
    """a, b in 8 bits and as 64-bit matrices on the GPU (what 8 bits hold is what is compared with)."""
    a, w = X.quantize(data(rows, cols, 1).cuda()), data(outs, cols, 2).cuda()
    b = X.quantize_weights(w) if squares else X.quantize(w)
    full = lambda m: R.from_blocks(m.values.cpu(), m.scales.cpu())  # noqa: E731
    return a, b, full(a).cuda(), (R.from_squares(b.values.cpu(), b.scales.cpu()) if squares else full(b)).cuda()


def limit(A, O, exact, dtype, want):
    """bounds() of the smaller sizes, on the GPU, in 32-bit magnitudes (1.001: their own rounding)."""
    per = (4 * 6 + 4 + A.shape[1] // 128) * 2 * R.U + (0.0 if exact else 7 * 2.0 ** -14)
    m = (A.abs().float() @ O.abs().float().t()).double() * 1.001
    return m * per + ROUNDING[dtype] * want.abs() + (6e-8 if dtype == torch.float16 else 1e-38)


def check(X, rows, outs, cols, squares, exact, form):
    a, b, A, O = operands(X, rows, outs, cols, squares)
    assert B.asgd_block_product_form(a._c, b._c, B.PRODUCT_ALL, int(exact), None) == form
    want = A @ O.t()
    for dtype in TYPES:
        y = X.product(a, b, dtype, exact=exact).double()
        assert ((y - want).abs() <= limit(A, O, exact, dtype, want)).all()
        # rows that begin anywhere: six elements more a row, one element in, and what lies between them stays
        room = torch.full((rows, outs + 7), 7.0, dtype=dtype, device="cuda")
        part = room[:, 1:outs + 1]
        B.asgd_block_product(a._c, b._c, B.PRODUCT_ALL, int(exact), None, part.data_ptr(), X._type(dtype), outs + 7, X._stream(room))
        assert torch.equal(part.double(), y) and (room[:, 0] == 7).all() and (room[:, outs + 1:] == 7).all()


# several strips of eight tiles, the last of them short, and tiles that both ends cut; one block, an even and an odd number of them, a short last one
@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("squares", [True, False])
@pytest.mark.parametrize("rows,outs,cols", [(1500, 1500, 128), (1411, 1601, 300), (1537, 1500, 512), (2300, 1025, 1100)])
def test_tiles_of_128(X, rows, outs, cols, squares, exact):
    check(X, rows, outs, cols, squares, exact, B.PRODUCT_FORM_TILES_128)


@pytest.mark.parametrize("rows,outs,cols", [(4000, 3900, 128), (3300, 4800, 300), (4090, 4095, 512), (3841, 4001, 1150)])
def test_tiles_of_256(X, rows, outs, cols):
    check(X, rows, outs, cols, True, False, B.PRODUCT_FORM_TILES_256)


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("squares", [True, False])
@pytest.mark.parametrize("rows,outs,cols", [(33, 65, 128), (777, 301, 1100), (600, 190, 640), (100, 999, 2049)])
def test_tiles_of_64(X, rows, outs, cols, squares, exact):
    check(X, rows, outs, cols, squares, exact, B.PRODUCT_FORM_TILES_64)


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("squares", [True, False])
@pytest.mark.parametrize("rows,outs,cols", [(16, 1001, 4000), (17, 300, 1100), (32, 33, 100), (31, 33000, 128)])
def test_few_rows(X, rows, outs, cols, squares, exact):
    check(X, rows, outs, cols, squares, exact, B.PRODUCT_FORM_FEW)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,outs,cols", [(1500, 1601, 1300), (4000, 3900, 700)])
def test_a_layer_and_its_gradients(X, rows, outs, cols, dtype):
    """linear() and linear_backward() at sizes whose products take the large tiles."""
    x, w, d = data(rows, cols, 1, dtype), data(outs, cols, 2), data(rows, outs, 3, dtype)
    q, t = X.quantize_weights(w.cuda()), X.quantize_weights(w.cuda(), turned=True)
    y, kept = X.linear(x.cuda(), q, train=True)
    d_x, d_w = X.linear_backward(d.cuda(), kept, t)
    assert torch.equal(y, X.linear(x.cuda(), q))
    W = R.from_squares(*R.to_squares(w))[:, :cols].cuda()
    A, D = R.rounded(x.float()).cuda(), R.rounded(d.float()).cuda()
    Dt, At = R.rounded(d.float().t()).cuda(), R.rounded(x.float().t()).cuda()
    exact = dtype != torch.bfloat16
    for got, a, b, e, ty in ((y, A, W, exact, dtype), (d_x, D, W.t(), exact, dtype), (d_w, Dt, At, True, torch.float32)):
        want = a @ b.t()
        assert got.dtype == ty and ((got.double() - want).abs() <= limit(a, b, e, ty, want)).all()


@pytest.mark.parametrize("exact", [False, True])
def test_gathered_rows_far_apart(X, exact):
    """An a of more than 2^32 bytes whose rows one tile takes from both ends, in both sums, against 64 bits."""
    T, K, N, E = 280_000, 16_384, 24, 3
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    at = [0, 1, 140_000, 279_998, 279_999]
    x, w = data(5, K, 8), data(E * N, K, 2).view(E, N, K)
    few = X.quantize(x.cuda())
    values = torch.zeros((T, K), dtype=torch.uint8, device="cuda")
    scales = torch.ones((K // 128, T), device="cuda")
    values[at], scales[:, at] = few.values.view(torch.uint8), few.scales
    a, b = X.Blocks(values, scales, K, squares=False), X.quantize_weights(w.cuda())
    ids = torch.zeros((T, 1), dtype=torch.int32, device="cuda")
    ids[2:140_000] = 1
    ids[140_001:279_998] = 1
    order = X.plan(ids, E)
    assert B.asgd_block_product_form(a._c, b._c, B.PRODUCT_GATHER, int(exact), order._c) == B.PRODUCT_FORM_TILES_128_FAR
    y = X.product(a, b, torch.float32, order, gather=True, exact=exact)
    A, O = R.from_blocks(few.values.cpu(), few.scales.cpu()).cuda(), R.from_squares(b.values[0].cpu(), b.scales[0].cpu()).cuda()
    want = A @ O.t()
    got = y[order.places[at].long()].double()
    assert ((got - want).abs() <= limit(A, O, exact, torch.float32, want)).all() and int((y.abs().sum(1) > 0).sum()) == 5


@pytest.mark.parametrize("T,k,E", [(140_000, 8, 256), ((1 << 20) + 5, 1, 1000), (1 << 19, 4, 9)])
def test_order_of_more_than_a_million_slots(X, T, k, E):
    """Workgroups that take several rounds of slots each."""
    g = torch.Generator().manual_seed(k)
    ids = torch.randint(-1, E, (T, k), generator=g).int()
    ids[1000:2000] = -1
    p = X.plan(ids.cuda(), E)
    flat = ids.reshape(-1).long()
    used, counts = int((flat >= 0).sum()), torch.bincount(flat[flat >= 0], minlength=E)
    offsets = torch.cat([torch.zeros(1, dtype=torch.long), torch.cumsum(counts, 0)])
    blocks = torch.cat([torch.zeros(1, dtype=torch.long), torch.cumsum((counts + 127) // 128, 0)])
    slots = torch.argsort(torch.where(flat < 0, torch.full_like(flat, E), flat), stable=True)
    places = torch.empty_like(slots)
    places[slots] = torch.arange(len(slots))
    places[flat < 0] = -1
    slots[used:] = -1
    assert torch.equal(p.offsets.cpu().long(), offsets) and torch.equal(p.blocks.cpu().long(), blocks)
    assert torch.equal(p.slots.cpu().long(), slots) and torch.equal(p.places.cpu().long(), places)


@pytest.mark.parametrize("exact", [False, True])
def test_many_rows_of_unequal_experts(X, exact):
    """Strips of tiles that cross from one expert to the next, an expert without rows, one with a single row, tiles that end inside."""
    T, k, E, N, K = 3000, 2, 6, 1100, 700
    g = torch.Generator().manual_seed(5)
    ids = torch.randint(0, 3, (T, k), generator=g).int()
    ids[17, 0], ids[:, 1] = 5, torch.where(torch.rand(T, generator=g) < 0.2, -1, 3).int()
    x, w = data(T, K, 1), data(E * N, K, 2).view(E, N, K)
    a, b, order = X.quantize(x.cuda()), X.quantize_weights(w.cuda()), X.plan(ids.cuda(), E)
    assert B.asgd_block_product_form(a._c, b._c, B.PRODUCT_GATHER, int(exact), order._c) == B.PRODUCT_FORM_TILES_128
    y = X.product(a, b, torch.float32, order, gather=True, exact=exact)
    by_place = X.product(X.quantize(x.cuda(), plan=order), b, torch.float32, order, exact=exact)
    A, places = R.rounded(x).cuda(), order.places.cpu().view(T, k)
    for e in range(E):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if len(t):
            O = R.from_squares(b.values[e].cpu(), b.scales[e].cpu()).cuda()[:, :K]
            want, at = A[t] @ O.t(), places[t, j].long().cuda()
            for got in (y, by_place):
                assert ((got[at].double() - want).abs() <= limit(A[t], O, exact, torch.float32, want)).all()
