"""Refusals of the layers in rows of signed codes that come before any work, and so need no GPU."""
import pytest
import torch

from paper_2506_17974_b200 import training as tr


@pytest.mark.parametrize("x,residual", [(torch.bfloat16, torch.float16), (torch.float16, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_residual_of_another_type(x, residual):
    """The output has the residual's type, and the gradients of x and the weight x's: with two types the backward pass would be refused."""
    with pytest.raises(ValueError, match="residual"):
        tr.linear_rows8_layer(torch.ones(2, 32, dtype=x), torch.ones(4, 32), residual=torch.ones(2, 4, dtype=residual))
