"""What the tensor calls of the routed experts refuse beyond shapes: other 8-bit types, changed structures, other devices, gradients that
would be lost.  No GPU is needed."""
import pytest
import torch

from paper_1505_04956_amd import binding as B
from paper_1505_04956_amd import experts as X


@pytest.mark.parametrize("dtype", [torch.float8_e5m2, torch.float8_e4m3fnuz, torch.float8_e5m2fnuz, torch.int8, torch.bool])
def test_bytes_of_other_types_are_refused(dtype):
    """Their bytes would be read as e4m3 numbers."""
    for values, scales in ((torch.zeros(4, 128, dtype=torch.uint8).view(dtype), torch.zeros(1, 1)),
                           (torch.zeros(2, 4, 128, dtype=torch.uint8).view(dtype), torch.zeros(2, 1, 1))):
        with pytest.raises(ValueError, match="values"):
            X.Blocks(values, scales, 100)
    for same in (torch.uint8, torch.float8_e4m3fn):
        assert X.Blocks(torch.zeros(4, 128, dtype=torch.uint8).view(same), torch.zeros(1, 1), 100).rows == 4


def test_structures_do_not_change():
    """The library reads sizes and addresses that were taken when they were made: with a smaller rule.k the ids of route() would be written
    beyond their end, with other w.values the old ones be read after they are freed."""
    rule, plan = X.Rule(4), X.Plan(5, 2, 3, "cpu")
    w = X.Blocks(torch.zeros(2, 4, 128, dtype=torch.uint8), torch.zeros(2, 1, 1), 100)
    rows = X._Rows(torch.zeros(3, 100), False, None)
    kept = X.Kept(plan, torch.zeros(5, 2), torch.zeros(10, 4), rows)
    for thing, names in ((rule, ("k",)), (plan, ("T", "k", "E", "offsets", "blocks", "slots", "places")),
                         (w, ("values", "scales", "rows", "cols", "count", "squares")), (rows, ("memory", "rows", "cols")),
                         (kept, ("plan", "weights", "y", "x_turned"))):
        for name in names:
            was = getattr(thing, name)
            with pytest.raises(AttributeError):
                setattr(thing, name, was)
            assert getattr(thing, name) is was or getattr(thing, name) == was
        with pytest.raises(AttributeError):
            thing.other = 1
    assert (rule.k, plan.T, plan.k, plan.E, w.rows, w.cols, w.count, w.squares) == (4, 5, 2, 3, 4, 100, 2, True)
    assert plan.offsets.numel() == plan.blocks.numel() == 4 and plan.slots.numel() == plan.places.numel() == 10


class Elsewhere(torch.Tensor):
    """A tensor on the CPU that says it is on the GPU, or (`there`) on another one."""
    there = 0

    def get_device(self):
        return self.there


class OnAnother(Elsewhere):
    there = 1


def test_a_plan_on_another_device_is_refused(monkeypatch):
    """Its addresses would be read by kernels of the tensors' device.  (Nothing gets as far as a kernel here: what calls the library is replaced.)"""
    for name in ("asgd_block_quantize", "asgd_block_quantize_both", "asgd_block_product", "asgd_experts_sum", "asgd_experts_sum_backward"):
        monkeypatch.setattr(B, name, lambda *a: None)
    monkeypatch.setattr(X, "_stream", lambda t: 0)
    monkeypatch.setattr(X, "_raw_stream", lambda index: 0)
    with monkeypatch.context() as m:
        empty = torch.empty
        m.setattr(torch, "empty", lambda *a, **k: empty(*a, **k).as_subclass(OnAnother))
        plan = X.Plan(8, 2, 3, "cpu")
    assert plan.offsets.get_device() == 1
    here = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype).as_subclass(Elsewhere)  # noqa: E731
    x, y, d = here(8, 200), here(16, 40), here(8, 40)
    w = X.Blocks(here(3, 40, 256, dtype=torch.uint8), here(3, 1, 2), 200)
    a, turned = X.Blocks(here(16, 256, dtype=torch.uint8), here(2, 16), 200, squares=False), X.Blocks(here(40, 384, dtype=torch.uint8), here(3, 40), 384, squares=False)
    for call in (lambda: X.quantize(x, plan=plan), lambda: X.quantize(x, turned=True, plan=plan), lambda: X._quantized(x, plan=plan), lambda: X._quantized_both(x, plan),
                 lambda: X.product(a, w, torch.float32, plan), lambda: X.product_over(turned, turned, plan), lambda: X.experts_sum(y, plan, torch.float32),
                 lambda: X.experts_sum_backward(d, y, plan)):
        with pytest.raises(ValueError, match="tensors on"):
            call()


def calls_that_lose_gradients(wanted):
    """Every call with each of its inputs that can have a gradient; wanted(t) gives it one."""
    x, l, i = torch.zeros(4, 128), torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    c, rule, plan = torch.zeros(4, 2), X.Rule(2), X.Plan(4, 2, 3, "cpu")
    w = X.Blocks(torch.zeros(3, 6, 128, dtype=torch.uint8), torch.zeros(3, 1, 1), 128)
    one = X.Blocks(torch.zeros(6, 128, dtype=torch.uint8), torch.zeros(1, 1), 128)
    back, all_back = X.Blocks(torch.zeros(128, 128, dtype=torch.uint8), torch.zeros(1, 1), 6), X.Blocks(torch.zeros(3, 128, 128, dtype=torch.uint8), torch.zeros(3, 1, 1), 6)
    y, d = torch.zeros(8, 6), torch.zeros(4, 6)
    of_x = X._Rows(x, True, None)
    kept = X.Kept(plan, c, y, X._Rows(x, True, plan))
    return [lambda: X.route(wanted(l), rule), lambda: X.route(l, rule, bias=wanted(torch.zeros(8))), lambda: X.route_backward(wanted(l), rule, i, c),
            lambda: X.route_backward(l, rule, i, wanted(c)), lambda: X.route_backward(l, rule, i, c, bias=wanted(torch.zeros(8))),
            lambda: X.Blocks(torch.zeros(6, 128, dtype=torch.uint8), wanted(torch.zeros(1, 1)), 128),
            lambda: X.quantize(wanted(x)), lambda: X.quantize(x, plan=plan, weights=wanted(c)), lambda: X.quantize_weights(wanted(x)),
            lambda: X.quantize_weights(wanted(torch.zeros(2, 3, 4)), turned=True), lambda: X.experts_sum(wanted(y), plan, torch.float32),
            lambda: X.experts_sum(y, plan, torch.float32, weights=wanted(c)), lambda: X.experts_sum_backward(wanted(d), y, plan),
            lambda: X.experts_sum_backward(d, wanted(y), plan), lambda: X.linear(wanted(x), one), lambda: X.linear(wanted(x), one, train=True),
            lambda: X.linear(wanted(torch.zeros(40, 128)), one), lambda: X.linear_backward(wanted(d), of_x, back), lambda: X.experts(wanted(x), i, c, w),
            lambda: X.experts(x, i, wanted(c), w), lambda: X.experts(wanted(x), i, c, w, train=True), lambda: X.experts_backward(wanted(d), kept, all_back)]


def test_gradients_that_would_be_lost_are_refused():
    """The results have no history: a tensor that wants a gradient is to be detached, or used where none are recorded."""
    for call in calls_that_lose_gradients(lambda t: t.clone().requires_grad_(True)):
        with pytest.raises(ValueError, match="gradient"):
            call()
    with torch.no_grad():
        for call in calls_that_lose_gradients(lambda t: t.clone().requires_grad_(True))[:5]:
            with pytest.raises(ValueError, match="no CPU fallback"):
                call()
    for call in calls_that_lose_gradients(lambda t: t.clone().requires_grad_(True).detach())[:5]:
        with pytest.raises(ValueError, match="no CPU fallback"):
            call()


def test_tangents_that_would_be_lost_are_refused():
    from torch.autograd import forward_ad
    with forward_ad.dual_level():
        for call in calls_that_lose_gradients(lambda t: forward_ad.make_dual(t, torch.ones_like(t))):
            with pytest.raises(ValueError, match="gradient"):
                call()


def test_which_kernel_a_product_takes():
    """From sizes and forms alone: nothing is enqueued, addresses are not used."""
    def blocks(rows, cols, form=B.BLOCKS_ROWS, count=1, **over):
        return B.asgd_blocks(1 << 20, None if form == B.BLOCKS_RAW else 1 << 20, rows, cols, form, count, over.get("type", 0), over.get("stride", 0))

    def form(rows, outs, cols, exact=0, squares=B.BLOCKS_SQUARES):
        return B.asgd_block_product_form(blocks(rows, cols), blocks(outs, cols, squares), B.PRODUCT_ALL, exact, None)
    assert form(32, 4096, 4096) == B.PRODUCT_FORM_FEW and form(33, 4096, 4096) == B.PRODUCT_FORM_TILES_64
    assert form(777, 1001, 1100) == B.PRODUCT_FORM_TILES_64 and form(65536, 1024, 128, 1) == B.PRODUCT_FORM_TILES_128
    assert form(8192, 8192, 8192) == B.PRODUCT_FORM_TILES_256 and form(8192, 8192, 8192, 1) == B.PRODUCT_FORM_TILES_128
    assert form(8192, 8192, 8192, 0, B.BLOCKS_ROWS) == B.PRODUCT_FORM_TILES_128
    assert form(0, 8, 8) == B.PRODUCT_FORM_NONE and form(8, 0, 8) == B.PRODUCT_FORM_NONE and form(8, 8, 8, 2) == B.PRODUCT_FORM_NONE
    raw = blocks(16, 200, B.BLOCKS_RAW, stride=200)
    assert B.asgd_block_product_form(raw, blocks(8, 200, B.BLOCKS_SQUARES), B.PRODUCT_ALL, 0, None) == B.PRODUCT_FORM_FEW
    assert B.asgd_block_product_form(raw, blocks(8, 200), B.PRODUCT_ALL, 0, None) == B.PRODUCT_FORM_NONE

    def experts(T, k, E, cols, mode=B.PRODUCT_GATHER):
        o = B.asgd_route_order(T, k, E, *[1 << 20] * 4)
        if mode == B.PRODUCT_OVER:
            cols = X.BLOCK * B.asgd_route_max_blocks(T, k, E)
            return B.asgd_block_product_form(blocks(64, cols), blocks(96, cols), mode, 1, o)
        return B.asgd_block_product_form(blocks(T if mode == B.PRODUCT_GATHER else T * k, cols), blocks(96, cols, B.BLOCKS_SQUARES, E), mode, 0, o)
    assert experts(24, 5, 100, 1000) == B.PRODUCT_FORM_FEW and experts(4093, 4, 64, 2048) == B.PRODUCT_FORM_TILES_128
    assert experts(280_000, 1, 3, 16_384) == B.PRODUCT_FORM_TILES_128_FAR and experts(4093, 4, 64, 2048, B.PRODUCT_PLACES) == B.PRODUCT_FORM_TILES_128
    assert experts(4, 1, 64, 0, B.PRODUCT_OVER) == B.PRODUCT_FORM_TILES_128
