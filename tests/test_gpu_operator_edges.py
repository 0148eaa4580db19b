"""Sizes of nothing."""
import pytest
import torch

from paper_2607_23115_gb300 import fp8

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.mark.parametrize("shape", [(0,), (6, 0), (2, 3, 0), (0, 3, 0), (40, 5, 0)])
def test_no_columns(shape):
    """Sums of nothing are zeros."""
    w = fp8.quantize_weight(torch.zeros(130, 0, device=DEV), grad=True)
    x = torch.zeros(shape, device=DEV)
    y = fp8.linear(x, w)
    assert y.shape == (*shape[:-1], 130) and not y.any()
    dx, dw = fp8.linear_grad(torch.randn_like(y), x, w)
    assert dx.shape == shape and dw.shape == (130, 0)
