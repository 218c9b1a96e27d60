"""Gradients whose dY is at the end of the type's range, or not finite: g = dropout(dY) a'(Z)
may pass the range of fp16 where dX and dW are in it."""
import pytest
import torch

from tests import layers_ref as R
from tests.test_gpu_dropout import _rng, mlp  # noqa: F401

pytestmark = pytest.mark.gpu

# few rows (second values of g), more of them, tiles, narrow layers, deep and odd ones
SHAPES = [(4, 64, 96), (40, 72, 200), (64, 33, 1001), (65, 40, 120), (300, 136, 264), (3, 50, 5), (64, 7, 96),
          (200, 64, 3), (500, 520, 520)]


def _tensors(rows, d_in, d_out, dtype, size):
    """Inputs of which dX and dW are in fp16's range for |dY| up to `size`."""
    g = torch.Generator().manual_seed(rows + d_out)
    dt = R.DTYPES[dtype]
    X = torch.randn(rows, d_in, generator=g).mul_(0.3 / rows ** 0.5 * 0.1).to(dt)
    W = torch.randn(d_in, d_out, generator=g).mul_(0.3 / d_out ** 0.5 * 0.1).to(dt)
    Z = torch.randn(rows, d_out, generator=g).to(dt)
    dY = (torch.rand(rows, d_out, generator=g) * 0.5 + 0.5).mul_(size)
    dY = torch.where(torch.rand(rows, d_out, generator=g) < 0.5, dY, -dY).to(dt)
    return [t.cuda() for t in (X, W, Z, dY)]


@pytest.mark.parametrize("rows,d_in,d_out", SHAPES)
@pytest.mark.parametrize("act,p", [("gelu", 0.0), ("relu", 0.1), ("none", 0.5), ("silu", 0.5), ("gelu_tanh", 0.9)])
def test_large_gradients_in_fp16(mlp, rows, d_in, d_out, act, p):  # noqa: F811
    """|dY| of 32,752 to 65,504: g is up to 1.13 / q times that."""
    print(rows, d_in, d_out, act, p, flush=True)
    X, W, Z, dY = _tensors(rows, d_in, d_out, "f16", 65504.0)
    ctx = mlp.mlp_linear_init(W, None, act, max_rows=rows)
    dx, dw, _ = mlp.mlp_linear_backward(ctx, X, dY, z=None if act == "none" else Z, p=p, rng=_rng(9, 2))
    torch.cuda.synchronize()
    ref, bound = R.backward(X, W, Z, dY, act, p, (9, 2), "f16")
    assert float(ref["g"].abs().max()) > 65504 or rows * d_out < 64   # (a few g may all be small)
    assert float(ref["dx"].abs().max()) < 60000 and float(ref["dw"].abs().max()) < 60000
    R.check("dx", dx, ref["dx"], bound["dx"])
    R.check("dw", dw, ref["dw"], bound["dw"])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,d_in,d_out", SHAPES)
@pytest.mark.parametrize("act,p", [("none", 0.5), ("silu", 0.1), ("gelu", 0.0)])
def test_infinite_gradients(mlp, dtype, rows, d_in, d_out, act, p):  # noqa: F811
    """One infinity and one NaN in dY: as in the formula, infinities of the sign of W and X in
    one row of dX and one column of dW, NaN in another, the rest as without them."""
    print(dtype, rows, d_in, d_out, act, p, flush=True)
    X, W, Z, dY = _tensors(rows, d_in, d_out, dtype, 1.0)
    Z[:, 1:3] = 0.5                      # a'(z) > 0
    keep = torch.from_numpy(R.keep_mask(9, 2, rows, d_out, p)) if p else torch.ones(rows, d_out, dtype=torch.bool)
    r1 = int(keep[:, 1].nonzero()[0])
    left = keep[:, 2].clone()
    left[r1] = False
    r2 = int(left.nonzero()[0])
    dY[r1, 1], dY[r2, 2] = float("-inf"), float("nan")
    ctx = mlp.mlp_linear_init(W, None, act, max_rows=rows)
    dx, dw, _ = mlp.mlp_linear_backward(ctx, X, dY, z=None if act == "none" else Z, p=p, rng=_rng(9, 2))
    torch.cuda.synchronize()
    assert torch.equal(dx[r1], torch.where(W[:, 1] > 0, float("-inf"), float("inf")).to(dx.dtype))
    assert torch.equal(dw[:, 1], torch.where(X[r1] > 0, float("-inf"), float("inf")).to(dw.dtype))
    assert bool(dx[r2].isnan().all()) and bool(dw[:, 2].isnan().all())
    dY[r1, 1] = dY[r2, 2] = 0
    ref, bound = R.backward(X, W, Z, dY, act, p, (9, 2), dtype)
    rows_left = [r for r in range(rows) if r not in (r1, r2)]
    cols_left = [c for c in range(d_out) if c not in (1, 2)]
    R.check("dx", dx[rows_left], ref["dx"][rows_left], bound["dx"][rows_left])
    R.check("dw", dw[:, cols_left], ref["dw"][:, cols_left], bound["dw"][:, cols_left])
