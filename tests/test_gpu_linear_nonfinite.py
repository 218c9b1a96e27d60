"""Infinities and NaN in X and W: in the rows and columns of the results where the formula
has them, and nowhere else, by every kernel."""
import pytest
import torch

from tests import layers_ref as R
from tests.test_gpu_dropout import _rng, _rows, mlp  # noqa: F401
from tests.test_gpu_linear import _layer

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
# narrow (with and without matrix instructions), few rows with and without splits, odd and whole tiles, splits
SHAPES = [(5, 1032, 3), (70, 24, 5), (300, 6, 200), (4, 4096, 264), (33, 40, 131), (64, 264, 264), (130, 777, 1001),
          (600, 520, 520), (2100, 136, 264)]


def _all_infinite(t, signs, parts):
    """t is signs' infinity. parts: or NaN, where an operand is a sum of parts (three of an
    fp32 value, two of g up to 64 rows or of fewer than eight outputs): inf (a + b) is taken as inf a + inf b, which is NaN
    where b is 0 or of another sign."""
    want = torch.where(signs > 0, INF, -INF).to(t.dtype)
    return bool(((t == want) | t.isnan()).all()) if parts else torch.equal(t, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,d_in,d_out", SHAPES)
def test_forward(mlp, dtype, rows, d_in, d_out):  # noqa: F811
    print(dtype, rows, d_in, d_out, flush=True)
    g = torch.Generator().manual_seed(rows)
    W, b = _layer(g, d_in, d_out, dtype, True)
    _, x = _rows(g, rows, d_in, dtype, 1)
    ctx = mlp.mlp_linear_init(W, b, "none", max_rows=rows)
    k = d_in - 1
    bad_rows, bad_cols = [1, rows - 1], [0, d_out - 1]
    x[1, k], x[rows - 1, 0] = -INF, NAN
    y = mlp.mlp_linear_forward(ctx, x)
    parts = dtype == "f32"
    assert _all_infinite(y[1], -W[k], parts) and bool(y[rows - 1].isnan().all())
    x[1, k] = x[rows - 1, 0] = 0.25
    ref, _, bound, _ = R.forward(x, W, b, None, "none", 0.0, None, dtype)
    left = [r for r in range(rows) if r not in bad_rows]
    R.check("rows", y[left], ref[left], bound[left])
    W[k, 0], W[1, d_out - 1] = INF, NAN
    y = mlp.mlp_linear_forward(ctx, x)
    assert _all_infinite(y[:, 0], x[:, k], parts) and bool(y[:, d_out - 1].isnan().all())
    left = [c for c in range(d_out) if c not in bad_cols]
    R.check("columns", y[:, left], ref[:, left], bound[:, left])
    # what ReLU masks is 0, an infinity or not; a NaN passes; what dropout drops is 0
    relu = mlp.mlp_linear_init(W, b, "relu", max_rows=rows)
    keep = torch.from_numpy(R.keep_mask(3, 4, rows, d_out, 0.5)).cuda()
    y = mlp.mlp_linear_forward(relu, x, p=0.5, rng=_rng(3, 4))
    assert bool((y[~keep] == 0).all()) and bool(y[:, d_out - 1][keep[:, d_out - 1]].isnan().all())
    if dtype != "f32":
        assert bool((y[:, 0][keep[:, 0]] == torch.where(x[:, k] > 0, INF, 0.0)[keep[:, 0]]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,d_in,d_out", SHAPES)
def test_backward(mlp, dtype, rows, d_in, d_out):  # noqa: F811
    print(dtype, rows, d_in, d_out, flush=True)
    g = torch.Generator().manual_seed(rows)
    W, b = _layer(g, d_in, d_out, dtype, True)
    _, x = _rows(g, rows, d_in, dtype, 0)
    _, z = _rows(g, rows, d_out, dtype, 1)
    _, dy = _rows(g, rows, d_out, dtype, 0)
    z[1, :] = 0.5
    z[:, d_out - 1] = 0.5       # a'(z) > 0 where it is multiplied with what is not finite
    ref, bound = R.backward(x, W, z, dy, "silu", 0.0, None, dtype)
    ctx = mlp.mlp_linear_init(W, b, "silu", max_rows=rows)
    # X is in dW alone, by rows; W in dX alone, by columns
    x[1, 0], x[0, d_in - 1] = INF, NAN
    W[0, d_out - 1], W[1, 0] = -INF, NAN
    dx, dw, db = mlp.mlp_linear_backward(ctx, x, dy, z=z)
    torch.cuda.synchronize()
    parts = dtype == "f32" or rows <= 64 or d_out < 8
    assert _all_infinite(dw[0], dy[1], parts) and bool(dw[d_in - 1].isnan().all())
    assert _all_infinite(dx[:, 0], -dy[:, d_out - 1], parts) and bool(dx[:, 1].isnan().all())
    left = [i for i in range(d_in) if i not in (0, d_in - 1)]
    R.check("dw", dw[left], ref["dw"][left], bound["dw"][left])
    left = list(range(2, d_in))
    R.check("dx", dx[:, left], ref["dx"][:, left], bound["dx"][:, left])
    R.check("db", db, ref["db"], bound["db"])
