"""nn.gated_linear without a GPU: refusals."""
import math

import pytest
import torch
import torch.autograd.forward_ad as fwad

from paper_2202_13808_amd import nn as dnn


@pytest.mark.parametrize("gamma", [-0.5, 1.5, math.nan, -math.inf])
def test_gated_linear_refuses_rates_that_are_none(gamma):
    x, w = torch.randn(2, 8), torch.randn(6, 8)
    for weight in (w, w.clone().requires_grad_(True)):
        with pytest.raises(ValueError, match="gamma"):
            dnn.gated_linear(x, weight, gamma=gamma)
    assert dnn.gated_linear(x, w, gamma=0.0).shape == (2, 3) and dnn.gated_linear(x, w, gamma=1.0).shape == (2, 3)


def test_dual_tensors_transforms_and_traces_are_noticed():
    x = torch.ones(3)
    assert not dnn._followed(x, None, x)
    with fwad.dual_level():
        dual = fwad.make_dual(x, x)
        assert dnn._followed(x, dual) and dnn._followed(dual, None) and not dnn._followed(x, None)
        with torch.no_grad():
            assert dnn._followed(dual)
    assert not dnn._followed(x)
    seen = []
    torch.func.jvp(lambda t: seen.append(dnn._followed(t)) or t, (x,), (x,))
    torch.func.vmap(lambda t: seen.append(dnn._followed(t)) or t)(x)
    torch.jit.trace(lambda t: seen.append(dnn._followed(t)) or t + 1, (x,), check_trace=False)
    assert seen == [True, True, True] and not dnn._followed(x)
