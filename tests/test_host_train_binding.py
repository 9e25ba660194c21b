"""What the binding of the training operators refuses before it reaches the library.  Needs no GPU."""
import pytest
import torch

from paper_2311_12023_amd import lq


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int64, "fp32", None])
def test_workspaces_of_other_types(dtype):
    with pytest.raises(TypeError):
        lq.cross_entropy_workspace(4, 64, 100, dtype)
    with pytest.raises(TypeError):
        lq.adapter_workspace(4, 64, 128, 8, dtype)
