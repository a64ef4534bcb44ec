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
