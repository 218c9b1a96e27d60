"""The largest widths and rows there are, next to the smallest."""
import pytest
import torch

from tests import layers_ref as R
from tests.test_gpu_dropout import _rng, _rows, mlp  # noqa: F401
from tests.test_gpu_linear import _layer

pytestmark = pytest.mark.gpu

M = 1 << 20


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,d_in,d_out", [(M, 9, 8), (M, 2, 1), (M - 1, 1, 17), (3, M, 9), (40, M, 3), (70, M - 1, 8), (5, 9, M),
                                             (40, 8, M - 3), (70, 3, M)])
def test_largest(mlp, dtype, rows, d_in, d_out):  # noqa: F811
    print(dtype, rows, d_in, d_out, flush=True)
    g = torch.Generator().manual_seed(d_in)
    W, b = _layer(g, d_in, d_out, dtype, True)
    _, x = _rows(g, rows, d_in, dtype, 0)
    _, z = _rows(g, rows, d_out, dtype, 0)
    _, dy = _rows(g, rows, d_out, dtype, 0)
    ctx = mlp.mlp_linear_init(W, b, "relu", max_rows=rows)
    y = mlp.mlp_linear_forward(ctx, x, p=0.5, rng=_rng(1, 2))
    dx, dw, db = mlp.mlp_linear_backward(ctx, x, dy, z=z, p=0.5, rng=_rng(1, 2))
    torch.cuda.synchronize()
    ry, _, by, _ = R.forward(x, W, b, None, "relu", 0.5, (1, 2), dtype)
    R.check("y", y, ry, by)
    ref, bound = R.backward(x, W, z, dy, "relu", 0.5, (1, 2), dtype)
    for n, t in (("dx", dx), ("dw", dw), ("db", db)):
        R.check(n, t, ref[n], bound[n])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 30_000_001), (30_000_001, 1), (3_000_000, 9)])
def test_largest_dropout(mlp, dtype, rows, cols):  # noqa: F811
    print(dtype, rows, cols, flush=True)
    x = torch.ones(rows, cols, dtype=R.DTYPES[dtype], device="cuda")
    y = mlp.mlp_dropout_forward(x, 0.25, _rng(4, 5))
    assert torch.equal(mlp.mlp_dropout_backward(x, 0.25, _rng(4, 5)), y)
    torch.cuda.synchronize()
    keep = torch.from_numpy(R.keep_mask(4, 5, rows, cols, 0.25))
    assert torch.equal(y.cpu() != 0, keep)
