"""Refusals of the layers' binding that need no GPU."""
import pytest
import torch

from paper_2606_30497_amd import mlp


def test_weights_that_are_not_on_a_gpu():
    for W in (torch.zeros(8, 16), torch.zeros(8, 16, dtype=torch.bfloat16)):
        with pytest.raises(TypeError):
            mlp.mlp_linear_init(W, None, "none", max_rows=8)
    with pytest.raises(TypeError):
        mlp.mlp_linear_init(torch.zeros(8, 16, dtype=torch.float64), None, "none", max_rows=8)
    with pytest.raises(ValueError):
        mlp.mlp_linear_init(torch.zeros(8), None, "none", max_rows=8)
