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
