"""What the binding of the dense layer takes and refuses beyond test_gpu_linear's refusals."""
import pytest
import torch

from tests.test_gpu_dropout import mlp  # noqa: F401

pytestmark = pytest.mark.gpu


def test_dw_of_another_layout(mlp):  # noqa: F811
    """A [d_out, d_in] dW (the layout of other frameworks' weights) has the right number of
    elements and would be filled with the transpose of its gradient."""
    W = torch.randn(16, 24, device="cuda")
    ctx = mlp.mlp_linear_init(W, None, "none", max_rows=8)
    x, dy = torch.randn(8, 16, device="cuda"), torch.randn(8, 24, device="cuda")
    want = mlp.mlp_linear_backward(ctx, x, dy)[1]
    for shape in ((24, 16), (1, 384), (16, 12, 2), (384, 1)):
        bad = torch.full(shape, 5.0, device="cuda")
        with pytest.raises(ValueError):
            mlp.mlp_linear_backward(ctx, x, dy, dW=bad)
        torch.cuda.synchronize()
        assert bool((bad == 5.0).all())
    flat = torch.empty(1000, device="cuda")
    for good in (torch.empty_like(W), flat[100:484]):
        assert mlp.mlp_linear_backward(ctx, x, dy, dW=good)[1] is good
        assert torch.equal(good.view(16, 24), want)
