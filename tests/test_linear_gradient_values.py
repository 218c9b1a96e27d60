"""Gradients of up to 64 rows in bf16 and fp16 take g = dropout(dY) a'(Z) unrounded, as two
values of the type (large products of 33 and more rows apart), at any widths, and so do those
of fewer than eight outputs at any rows: held to a bound without the rounding of g.

The bound, with u half a step of the type, e = 2^-24 and t half the type's smallest step:
- the two values leave at most u^2 |g| + t of an element of g (the second one's rounding);
  the products' n terms take it independently: 4 u^2 sqrt(sum (g w)^2) + t sum |w|.
- 2 n products are summed in fp32: 4 e sqrt(2 n + 32) sum |g w|, as in layers_ref.
- the activation's derivative: layers_ref's 16 e (1 + |z|) max(|z|, 1) |v| for each g.
- the result is rounded once: u |y|, or t.
"""
import math

import pytest
import torch

from tests import layers_ref as R

SMALLEST = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25}


def gradients(X, W, Z, dY, name, p, rng, dtype):
    """{"dx", "dw"}: (64-bit value, bound) for an unrounded g."""
    X, W, Z, dY = (None if t is None else t.detach().cpu().double() for t in (X, W, Z, dY))
    v = dY * R.factor(rng, dY.shape[0], dY.shape[1], p)
    g, eg = v, 4 * R.E * v.abs()
    if name != "none":
        g = v * R.act_grad(Z, name)
        eg = v.abs() * 16 * R.E * (1 + Z.abs()) * Z.abs().clamp(min=1)
    u, t = R.U[dtype], SMALLEST[dtype]
    out = {}
    for k, a, b, ea, eb in (("dx", g, W.t(), eg + t, None), ("dw", X.t(), g, None, eg + t)):
        y, S = a @ b, a.abs() @ b.abs()
        e = 4 * R.E * math.sqrt(2 * a.shape[1] + 32) * S + 4 * u * u * torch.sqrt((a * a) @ (b * b))
        e = e + (ea @ b.abs() if ea is not None else a.abs() @ eb)
        out[k] = y, e + u * (y.abs() + e) + t
    return out, g


def inputs(rows, d_in, d_out, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    dt = R.DTYPES[dtype]
    X, Z, dY = (torch.randn(rows, n, generator=gen).to(dt) for n in (d_in, d_out, d_out))
    return X, (torch.randn(d_in, d_out, generator=gen) * (2.0 / d_in) ** 0.5).to(dt), Z, dY


# rows, d_in, d_out: widths below eight on either side, both, odd ones, whole tiles, the
# largest products of 33 to 64 rows (2^28 terms)
SHAPES = [(1, 64, 1), (1, 1, 1), (2, 5, 7), (7, 1000, 3), (20, 7, 300), (32, 3, 3), (33, 257, 1), (40, 4099, 2),
          (64, 256, 1), (64, 1, 1000), (64, 5, 4100), (5, 24, 40), (16, 520, 264), (33, 512, 384), (48, 100, 1001),
          (64, 1032, 77), (64, 24, 5001), (40, 2560, 2600), (64, 4096, 1016), (64, 2048, 2040)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_bound_tells_a_rounded_g(dtype):
    """The bound refuses what a g of one value gives, or second values of wrong columns or
    rows, and has room for two values. (Not of fp16 sums of thousands of terms,
    whose fp32 roundings are granted more than what a rounded g adds.)"""
    u = R.DTYPES[dtype]
    for i, (rows, d_in, d_out) in enumerate(SHAPES):
        if rows * d_in * d_out > 1 << 27:
            continue
        X, W, Z, dY = inputs(rows, d_in, d_out, dtype, i)
        ref, g = gradients(X, W, Z, dY, "silu", 0.3, (5, i), dtype)
        hi = g.to(u).double()
        lo = (g - hi).to(u).double()
        for what, gg in (("one value", hi), ("other columns", hi + lo.roll(1, 1)), ("other rows", hi + lo.roll(1, 0)),
                         ("two values", hi + lo)):
            if what == "other columns" and d_out == 1 or what == "other rows" and rows == 1:
                continue
            for k, y, n in (("dx", gg @ W.double().t(), d_out), ("dw", X.double().t() @ gg, rows)):
                if n > 1024 and dtype == "f16" and what != "two values":
                    continue
                off = ((y.to(u).double() - ref[k][0]).abs() / ref[k][1]).max()
                # (a handful of results may all happen to be near)
                assert off <= 1 if what == "two values" else (off > 1 or y.numel() < 64), (what, k, rows, d_in, d_out, float(off))


@pytest.fixture(scope="module")
def mlp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_30497_amd import mlp as m
    m.load(require_built=True)
    return m


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,d_in,d_out", SHAPES)
def test_gradients_of_up_to_64_rows(mlp, dtype, rows, d_in, d_out):
    i = SHAPES.index((rows, d_in, d_out))
    X, W, Z, dY = (t.cuda() for t in inputs(rows, d_in, d_out, dtype, i))
    rng = torch.tensor([5, i], device="cuda")
    for act, p, most in (("silu", 0.3, rows), ("none", 0.5, rows + 300), ("relu", 0.0, 64)):
        print(dtype, rows, d_in, d_out, act, p, flush=True)
        ctx = mlp.mlp_linear_init(W, None, act, max_rows=most)
        z = None if act == "none" else Z
        dx, dw, _ = mlp.mlp_linear_backward(ctx, X, dY, z=z, p=p, rng=rng)
        torch.cuda.synchronize()
        ref, _ = gradients(X, W, z, dY, act, p, (5, i), dtype)
        R.check("dx", dx, *ref["dx"])
        R.check("dw", dw, *ref["dw"])
        # rows apart at odd strides, and each gradient alone: the same bits
        far = [torch.full((rows, t.shape[1] + 3), float("nan"), dtype=t.dtype, device="cuda")[:, :t.shape[1]].copy_(t)
               for t in (X, Z, dY)]
        z = None if act == "none" else far[1]
        assert torch.equal(mlp.mlp_linear_backward(ctx, None, far[2], z=z, p=p, rng=rng, need_dw=False)[0], dx)
        assert torch.equal(mlp.mlp_linear_backward(ctx, far[0], far[2], z=z, p=p, rng=rng, need_dx=False)[1], dw)


# 64 x 64 tiles, split and not, and 128 x 128 ones, by their number and for a deep product
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,d_in,d_out", [(65, 24, 1), (333, 777, 2), (1000, 64, 3), (3001, 40, 4), (700, 130, 5),
                                             (9000, 21, 6), (2100, 264, 7), (600, 1, 1), (130, 16500, 3), (3000, 2100, 5)])
def test_gradients_of_fewer_than_eight_outputs(mlp, dtype, rows, d_in, d_out):
    print(dtype, rows, d_in, d_out, flush=True)
    X, W, Z, dY = (t.cuda() for t in inputs(rows, d_in, d_out, dtype, rows))
    rng = torch.tensor([6, 7], device="cuda")
    ctx = mlp.mlp_linear_init(W, None, "gelu", max_rows=rows)
    dx, dw, _ = mlp.mlp_linear_backward(ctx, X, dY, z=Z, p=0.2, rng=rng)
    torch.cuda.synchronize()
    ref, _ = gradients(X, W, Z, dY, "gelu", 0.2, (6, 7), dtype)
    R.check("dx", dx, *ref["dx"])
    R.check("dw", dw, *ref["dw"])
    assert torch.equal(mlp.mlp_linear_backward(ctx, X, dY, z=Z, p=0.2, rng=rng, need_dx=False)[1], dw)
