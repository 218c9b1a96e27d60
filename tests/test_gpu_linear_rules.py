"""Few rows on either side of the rule between 16 and 32 rows a workgroup."""
import pytest
import torch

from tests import layers_ref as R
from tests.test_gpu_dropout import _rows, mlp  # noqa: F401
from tests.test_gpu_linear import _layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d_in,d_out", [(24, 4096, 2048), (20, 4096, 4096), (32, 4096, 4104), (17, 4099, 4101), (24, 8192, 4096), (31, 8200, 4104)])
def test_few_rows_of_wide_layers(mlp, dtype, rows, d_in, d_out):  # noqa: F811
    print(dtype, rows, d_in, d_out, flush=True)
    g = torch.Generator().manual_seed(d_out)
    W, b = _layer(g, d_in, d_out, dtype, True)
    _, x = _rows(g, rows, d_in, dtype, 0)
    _, dy = _rows(g, rows, d_out, dtype, 0)
    ctx = mlp.mlp_linear_init(W, b, "none", max_rows=rows)
    y = mlp.mlp_linear_forward(ctx, x)
    dx, _, _ = mlp.mlp_linear_backward(ctx, None, dy, need_dw=False, need_db=False)
    torch.cuda.synchronize()
    ry, _, by, _ = R.forward(x, W, b, None, "none", 0.0, None, dtype)
    R.check("y", y, ry, by)
    Wd, d = W.cpu().double(), dy.cpu().double()
    want, S = d @ Wd.t(), d.abs() @ Wd.abs().t()
    e = 4 * R.E * (d_out + 32) ** 0.5 * S
    R.check("dx", dx, want, e + R.U[dtype] * (want.abs() + e) + R.TINY[dtype])
