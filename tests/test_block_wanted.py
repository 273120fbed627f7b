"""Names of gradients that do not exist are refused, before anything else of a call is
looked at (CPU only)."""
import pytest
import torch

import paper_2607_10071_amd as fb


@pytest.mark.parametrize("want", [("wieght",), ("x", "residual"), "weight"])
def test_linear_backward(want):
    x, w, g = torch.zeros(2, 3), torch.zeros(4, 3), torch.zeros(2, 4)
    with pytest.raises(ValueError, match="want takes"):
        fb.linear_backward(g, x, w, want=want)
