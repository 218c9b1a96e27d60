"""Gradients of layers whose own shapes choose the larger tiles: dX by 256 x 128 tiles in fp32
and by 128 x 128 tiles of two stages in 16-bit types, dW by 256 x 128 tiles of a deep product
in fp32; odd tails in every direction."""
import pytest
import torch

from tests import layers_ref as R
from tests.test_gpu_dropout import _rng, _rows, mlp  # noqa: F401
from tests.test_gpu_linear import _layer

pytestmark = pytest.mark.gpu


# (dX: 400 tiles of 128 x 128 and more in fp32, over 256 in 16 bits with at most 128 of 256 x 256;
# dW: 1,024 tiles of 128 x 128 and more)
@pytest.mark.parametrize("dtype,rows,d_in,d_out", [("f32", 2600, 2601, 203), ("f32", 5003, 1300, 1029), ("f32", 1003, 4100, 4099),
                                                   ("f32", 130, 4224, 4100), ("bf16", 2400, 2700, 264), ("f16", 2399, 2701, 523),
                                                   ("bf16", 2305, 2304, 2312)])
def test_gradients_on_the_larger_tiles(mlp, dtype, rows, d_in, d_out):  # noqa: F811
    print(dtype, rows, d_in, d_out, flush=True)
    g = torch.Generator().manual_seed(rows)
    W, b = _layer(g, d_in, d_out, dtype, True)
    _, x = _rows(g, rows, d_in, dtype, 0)
    _, z = _rows(g, rows, d_out, dtype, 0)
    _, dy = _rows(g, rows, d_out, dtype, 0)
    ctx = mlp.mlp_linear_init(W, b, "gelu", max_rows=rows)
    dx, dw, db = mlp.mlp_linear_backward(ctx, x, dy, z=z, p=0.1, rng=_rng(1, 2))
    torch.cuda.synchronize()
    # 64 bits: of whole rows of dX, and of whole rows of dW (columns of X)
    keep = R.factor((1, 2), rows, d_out, 0.1)
    zd, dyd = z.cpu().double(), dy.cpu().double()
    v = dyd * keep
    gg = v * R.act_grad(zd, "gelu")
    eg = v.abs() * 16 * R.E * (1 + zd.abs()) * zd.abs().clamp(min=1)
    u, t = R.U[dtype], R.TINY[dtype]
    at = torch.randperm(rows, generator=g)[:40].tolist() + [0, rows - 1]
    cols = torch.randperm(d_in, generator=g)[:40].tolist() + [0, d_in - 1]
    Wd, xd = W.cpu().double(), x.cpu().double()
    for got, a, bb, ea, eb in ((dx[at], gg[at], Wd.t(), eg[at] + t, None), (dw[cols], xd[:, cols].t(), gg, None, eg + t)):
        want, S, n = a @ bb, a.abs() @ bb.abs(), a.shape[1]
        # as layers_ref.backward; the rounding of g to the type only where there is one
        e = 4 * R.E * (n + 32) ** 0.5 * S + (0 if dtype == "f32" else 4 * u * ((a * a) @ (bb * bb)).sqrt())
        e = e + (ea @ bb.abs() if ea is not None else a.abs() @ eb)
        R.check("sample", got, want, e + u * (want.abs() + e) + t)
    want = gg.sum(0)
    e = 4 * R.E * (rows + 32) ** 0.5 * gg.abs().sum(0) + eg.sum(0)
    R.check("db", db, want, e + u * (want.abs() + e) + t)
    # every element, against fp32 products on the GPU: rows or tiles left out are off by the whole
    gf, bar = gg.float().cuda(), 16 * u + 4 * R.E * (max(rows, d_in, d_out) + 32) ** 0.5
    for got, want in ((dx, gf @ W.float().t().contiguous()), (dw, x.float().t().contiguous() @ gf)):
        assert float((got.float() - want).norm() / want.norm()) <= bar
        assert float((got.float() - want).abs().max()) <= 8 * bar * float(want.abs().max())
