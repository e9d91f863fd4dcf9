"""nn.gated_linear without a GPU: refusals."""
import math

import pytest
import torch

from paper_2202_13808_amd import nn as dnn


@pytest.mark.parametrize("gamma", [-0.5, 1.5, math.nan, -math.inf])
def test_gated_linear_refuses_rates_that_are_none(gamma):
    x, w = torch.randn(2, 8), torch.randn(6, 8)
    for weight in (w, w.clone().requires_grad_(True)):
        with pytest.raises(ValueError, match="gamma"):
            dnn.gated_linear(x, weight, gamma=gamma)
    assert dnn.gated_linear(x, w, gamma=0.0).shape == (2, 3) and dnn.gated_linear(x, w, gamma=1.0).shape == (2, 3)
