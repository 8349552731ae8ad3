"""What the dense layers' modules make of the weights that they are given.  No GPU needed."""
import pytest
import torch

from paper_2302_03213_amd.dense import DenseLinear


@pytest.mark.parametrize("make", [lambda: torch.nn.Linear(8, 4).weight.t(), lambda: torch.randn(8, 1).expand(8, 4),
                                  lambda: torch.randn(8, 9)[:, 2:6], lambda: torch.randn(8, 4)])
def test_weights_of_any_strides(make):
    """Rows of W that are contiguous, as the calls want them, with values and memory of their own."""
    W, b = make(), torch.randn(8)[::2]
    layer = DenseLinear(W, b)
    assert layer.W.is_contiguous() and layer.bias.is_contiguous()
    assert torch.equal(layer.W, W) and torch.equal(layer.bias, b)
    assert layer.W.data_ptr() != W.data_ptr() and layer.W.requires_grad
