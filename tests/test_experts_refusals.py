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
