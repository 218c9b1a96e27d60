"""mlp_linear_forward / mlp_linear_backward against the 64-bit definition."""
import pytest
import torch

from tests import layers_ref as R
from tests.test_gpu_dropout import _rng, _rows, mlp  # noqa: F401

pytestmark = pytest.mark.gpu

# (rows, d_in, d_out, pad): one row to many, widths of one, odd ones, whole tiles
SHAPES = [(1, 1, 1, 0), (1, 32, 1, 0), (2, 5, 7, 3), (1, 256, 512, 0), (1, 1000, 1001, 1), (3, 2048, 40, 0),
          (8, 64, 4097, 0), (15, 777, 64, 2), (16, 512, 256, 8), (17, 33, 9, 0), (31, 1024, 130, 0), (32, 100, 264, 4),
          (33, 17, 2049, 5), (48, 520, 520, 0), (64, 256, 256, 0), (65, 255, 257, 0), (100, 1032, 72, 8),
          (128, 128, 128, 0), (129, 64, 1, 0), (200, 2056, 136, 0), (256, 512, 384, 0), (257, 96, 520, 16),
          (300, 513, 77, 1), (512, 1024, 256, 0), (1000, 40, 8, 0), (777, 136, 1000, 8), (1500, 8, 24, 0),
          (2000, 264, 264, 0), (40, 4104, 136, 0), (24, 130, 8200, 0), (1040, 1032, 2056, 0), (33, 4000, 4104, 0)]
# activation, p, bias, residual, z kept
OPTIONS = [("none", 0.0, False, False, False), ("relu", 0.0, True, True, True), ("gelu", 0.1, True, False, True),
           ("gelu_tanh", 0.5, False, True, False), ("silu", 0.3, True, True, True)]


def _layer(g, d_in, d_out, dtype, bias):
    W = (torch.randn(d_in, d_out, generator=g) * (2.0 / d_in) ** 0.5).to(R.DTYPES[dtype]).cuda()
    return W, (torch.randn(d_out, generator=g).to(R.DTYPES[dtype]).cuda() if bias else None)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,d_in,d_out,pad", SHAPES)
def test_forward(mlp, dtype, rows, d_in, d_out, pad):  # noqa: F811
    i = SHAPES.index((rows, d_in, d_out, pad)) + sorted(R.DTYPES).index(dtype)
    for act, p, bias, residual, keep_z in (OPTIONS[i % 5], OPTIONS[(i + 2) % 5]):
        print(dtype, rows, d_in, d_out, pad, act, p, bias, residual, keep_z, flush=True)
        g = torch.Generator().manual_seed(100 + i)
        W, b = _layer(g, d_in, d_out, dtype, bias)
        _, x = _rows(g, rows, d_in, dtype, pad, float("nan"))
        r = _rows(g, rows, d_out, dtype, pad, float("nan"))[1] if residual else None
        ybuf, y = _rows(g, rows, d_out, dtype, pad + 2)
        zbuf, z = _rows(g, rows, d_out, dtype, pad)
        ctx = mlp.mlp_linear_init(W, b, act, max_rows=rows)
        rng = (77, (1 << 32) - 5)
        mlp.mlp_linear_forward(ctx, x, residual=r, p=p, rng=_rng(*rng), out=y, z=z if keep_z else None)
        torch.cuda.synchronize()
        ry, rz, by, bz = R.forward(x, W, b, r, act, p, rng, dtype)
        R.check("y", y, ry, by)
        if keep_z:
            R.check("z", z, rz, bz)
        assert bool((ybuf[:, d_out:] == 7.0).all()) and bool((zbuf[:, d_out:] == 7.0).all())
        # contiguous tensors, and a second call, give the same bits
        y2 = mlp.mlp_linear_forward(ctx, x.contiguous(), residual=None if r is None else r.contiguous(), p=p,
                                    rng=_rng(*rng))
        assert torch.equal(y2, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,d_in,d_out,pad", SHAPES)
def test_backward(mlp, dtype, rows, d_in, d_out, pad):  # noqa: F811
    i = SHAPES.index((rows, d_in, d_out, pad)) + sorted(R.DTYPES).index(dtype)
    for act, p, bias, _, _ in (OPTIONS[i % 5], OPTIONS[(i + 3) % 5]):
        print(dtype, rows, d_in, d_out, pad, act, p, bias, flush=True)
        g = torch.Generator().manual_seed(200 + i)
        W, b = _layer(g, d_in, d_out, dtype, bias)
        _, x = _rows(g, rows, d_in, dtype, pad, float("nan"))
        _, z = _rows(g, rows, d_out, dtype, pad + 1, float("nan"))
        _, dy = _rows(g, rows, d_out, dtype, pad, float("nan"))
        dxbuf, dx = _rows(g, rows, d_in, dtype, pad + 3)
        ctx = mlp.mlp_linear_init(W, b, act, max_rows=rows)
        rng = (78, -3)
        _, dw, db = mlp.mlp_linear_backward(ctx, x, dy, z=None if act == "none" else z, p=p, rng=_rng(*rng), dX=dx)
        torch.cuda.synchronize()
        ref, bound = R.backward(x, W, z, dy, act, p, rng, dtype)
        R.check("dx", dx, ref["dx"], bound["dx"])
        R.check("dw", dw, ref["dw"], bound["dw"])
        assert bool((dxbuf[:, d_in:] == 7.0).all()) and (db is None) == (b is None)
        if db is not None:
            R.check("db", db, ref["db"], bound["db"])
        # each gradient alone, from contiguous tensors, and again: the same bits
        cx, cz, cdy = x.contiguous(), None if act == "none" else z.contiguous(), dy.contiguous()
        for need in ("dx", "dw", "db"):
            out = mlp.mlp_linear_backward(ctx, cx if need == "dw" else None, cdy, z=cz, p=p, rng=_rng(*rng),
                                          need_dx=need == "dx", need_dw=need == "dw", need_db=need == "db")
            for name, got, want in zip(("dx", "dw", "db"), out, (dx, dw, db)):
                assert (got is None) == (name != need or want is None)
                assert got is None or torch.equal(got, want), name


# shapes of the larger tiles (above 128 of 256 x 256, above 256 of 128 x 128), a depth that ends inside
# a chunk, row tails; whole activations on the CPU would take minutes, so the 64-bit
# reference is taken of a sample of rows and of columns
@pytest.mark.parametrize("dtype,rows,d_in,d_out", [("bf16", 3900, 136, 3600), ("f16", 3600, 3336, 300),
                                                   ("bf16", 3600, 4104, 3400), ("bf16", 2400, 264, 2700),
                                                   ("f32", 2600, 328, 2600), ("f32", 1100, 2600, 2650)])
def test_large_tiles(mlp, dtype, rows, d_in, d_out):  # noqa: F811
    g = torch.Generator().manual_seed(rows)
    W, b = _layer(g, d_in, d_out, dtype, True)
    _, x = _rows(g, rows, d_in, dtype, 0)
    _, z = _rows(g, rows, d_out, dtype, 0)
    _, dy = _rows(g, rows, d_out, dtype, 0)
    ctx = mlp.mlp_linear_init(W, b, "silu", max_rows=rows)
    y, zz = mlp.mlp_linear_forward(ctx, x, save_z=True)
    dx, dw, db = mlp.mlp_linear_backward(ctx, x, dy, z=z)
    torch.cuda.synchronize()
    at = torch.randperm(rows, generator=g)[:40].tolist() + [0, rows - 1]
    ry, rz, by, bz = R.forward(x[at], W, b, None, "silu", 0.0, None, dtype)
    R.check("y", y[at], ry, by)
    R.check("z", zz[at], rz, bz)
    ref, bound = R.backward(x[at], W, z[at], dy[at], "silu", 0.0, None, dtype)
    R.check("dx", dx[at], ref["dx"], bound["dx"])
    cols = torch.randperm(d_in, generator=g)[:24].tolist() + [0, d_in - 1]
    ref, bound = R.backward(x[:, cols], W[cols], z, dy, "silu", 0.0, None, dtype)
    R.check("dw", dw[cols], ref["dw"], bound["dw"])
    R.check("db", db, ref["db"], bound["db"])
    # every element, on the GPU in fp32: rows or tiles left out would be off by the whole
    u = 16 * R.U[dtype] + 4 * R.E * (max(rows, d_in, d_out) + 32) ** 0.5
    f = torch.nn.functional.silu(x.float() @ W.float() + b.float())
    assert float((y.float() - f).norm() / f.norm()) <= u and float((y.float() - f).abs().max()) <= 8 * u * float(f.abs().max())
    sg = torch.sigmoid(z.float())
    gg = dy.float() * sg * (1 + z.float() * (1 - sg))
    for got, want in ((dx, gg @ W.float().t()), (dw, x.float().t() @ gg)):
        assert float((got.float() - want).norm() / want.norm()) <= u
        assert float((got.float() - want).abs().max()) <= 8 * u * float(want.abs().max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows(mlp, dtype):  # noqa: F811
    g = torch.Generator().manual_seed(1)
    W, b = _layer(g, 40, 24, dtype, True)
    ctx = mlp.mlp_linear_init(W, b, "relu", max_rows=64)
    e = W.new_empty
    assert mlp.mlp_linear_forward(ctx, e(0, 40)).shape == (0, 24)
    dx, dw, db = mlp.mlp_linear_backward(ctx, e(0, 40), e(0, 24), z=e(0, 24), dW=torch.full_like(W, 3), db=torch.full_like(b, 3))
    assert dx.shape == (0, 40) and float(dw.abs().max()) == 0 and float(db.abs().max()) == 0


@pytest.mark.parametrize("rows", [1, 40, 600])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_dropout_of_the_layer_is_dropout(mlp, dtype, rows):  # noqa: F811
    """The layer's mask is that of mlp_dropout_forward with the same state and shape."""
    g = torch.Generator().manual_seed(2)
    W, b = _layer(g, 64, 203, dtype, True)
    _, x = _rows(g, rows, 64, dtype, 0)
    ctx = mlp.mlp_linear_init(W, b, "none", max_rows=rows)
    y = mlp.mlp_linear_forward(ctx, x, p=0.4, rng=_rng(3, 4))
    ones = torch.ones(rows, 203, device="cuda")
    assert torch.equal(y != 0, mlp.mlp_dropout_forward(ones, 0.4, _rng(3, 4)) != 0)
    # the backward call's too
    _, _, db = mlp.mlp_linear_backward(ctx, x, ones.to(W.dtype), p=0.4, rng=_rng(3, 4), need_dx=False, need_dw=False)
    ref = (torch.from_numpy(R.keep_mask(3, 4, rows, 203, 0.4)).double() * R.drop_scale(0.4)).sum(0)
    e = 4 * R.E * (rows + 32) ** 0.5 * ref + R.U[dtype] * ref
    R.check("db", db, ref, e)


def test_residual_in_place_and_masked_values(mlp):  # noqa: F811
    g = torch.Generator().manual_seed(3)
    W, b = _layer(g, 72, 48, "bf16", True)
    _, x = _rows(g, 130, 72, "bf16", 0)
    _, r = _rows(g, 130, 48, "bf16", 6)
    ctx = mlp.mlp_linear_init(W, b, "relu", max_rows=130)
    want = mlp.mlp_linear_forward(ctx, x, residual=r)
    got = mlp.mlp_linear_forward(ctx, x, residual=r, out=r)
    assert got is r and torch.equal(got, want)
    # gradients: what ReLU masks or dropout drops is 0, also where dY is not finite
    _, z = _rows(g, 130, 48, "bf16", 0)
    keep = torch.from_numpy(R.keep_mask(5, 6, 130, 48, 0.5)).cuda()
    dy = torch.where((z > 0) & keep, torch.randn(130, 48, device="cuda").to(z.dtype), torch.tensor(float("nan"), dtype=z.dtype, device="cuda"))
    dx, dw, db = mlp.mlp_linear_backward(ctx, x, dy, z=z, p=0.5, rng=_rng(5, 6))
    ref, bound = R.backward(x, W, z, torch.nan_to_num(dy), "relu", 0.5, (5, 6), "bf16")
    for n, t in (("dx", dx), ("dw", dw), ("db", db)):
        R.check(n, t, ref[n], bound[n])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_past_32_bits(mlp, dtype):  # noqa: F811
    """X, Y, Z and dY whose rows are so far apart that the last start past 2^32 bytes
    (fp32) and 2^31 elements."""
    rows, d_in, d_out, ld = 600, 40, 24, 1 << 22
    g = torch.Generator().manual_seed(4)
    W, b = _layer(g, d_in, d_out, dtype, True)

    def far(cols):
        t = torch.empty(rows * ld, dtype=W.dtype, device="cuda").view(rows, ld)[:, 8:8 + cols]
        t.copy_(torch.randn(rows, cols, generator=g))
        return t

    x, y, z, dy = far(d_in), far(d_out), far(d_out), far(d_out)
    ctx = mlp.mlp_linear_init(W, b, "silu", max_rows=rows)
    mlp.mlp_linear_forward(ctx, x, out=y, z=z)
    ry, rz, by, bz = R.forward(x, W, b, None, "silu", 0.0, None, dtype)
    R.check("y", y, ry, by)
    R.check("z", z, rz, bz)
    dx, dw, db = mlp.mlp_linear_backward(ctx, x, dy, z=z)
    ref, bound = R.backward(x, W, z, dy, "silu", 0.0, None, dtype)
    R.check("dx", dx, ref["dx"], bound["dx"])
    R.check("dw", dw, ref["dw"], bound["dw"])
    R.check("db", db, ref["db"], bound["db"])


def test_fewer_rows_than_the_context_has_room_for(mlp):  # noqa: F811
    g = torch.Generator().manual_seed(5)
    W, b = _layer(g, 264, 136, "bf16", True)
    big = mlp.mlp_linear_init(W, b, "gelu", max_rows=3000)
    for rows in (1, 20, 130, 700, 3000):
        _, x = _rows(g, rows, 264, "bf16", 0)
        _, dy = _rows(g, rows, 136, "bf16", 0)
        small = mlp.mlp_linear_init(W, b, "gelu", max_rows=rows)
        ry, rz, by, bz = R.forward(x, W, b, None, "gelu", 0.0, None, "bf16")
        for ctx in (big, small):
            y, z = mlp.mlp_linear_forward(ctx, x, save_z=True)
            R.check("y", y, ry, by)
            grads = mlp.mlp_linear_backward(ctx, x, dy, z=z)
            ref, bound = R.backward(x, W, z, dy, "gelu", 0.0, None, "bf16")
            for n, t in zip(("dx", "dw", "db"), grads):
                R.check(n, t, ref[n], bound[n])


def _block_loss(mlp, ctx1, ctx2, x, dy, rng):  # noqa: F811
    """One residual block x + dropout(gelu(x W1 + b1) W2 + b2) forward and backward;
    returns y and the gradients, dx with the residual's."""
    h, z1 = mlp.mlp_linear_forward(ctx1, x, save_z=True)
    y = mlp.mlp_linear_forward(ctx2, h, residual=x, p=0.1, rng=rng)
    dh, dw2, db2 = mlp.mlp_linear_backward(ctx2, h, dy, p=0.1, rng=rng)
    dx, dw1, db1 = mlp.mlp_linear_backward(ctx1, x, dh, z=z1)
    return y, dx + dy, dw1, db1, dw2, db2


@pytest.mark.parametrize("rows,d,f", [(37, 96, 200), (400, 128, 512)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_residual_block_and_its_graph(mlp, dtype, rows, d, f):  # noqa: F811
    """Two layers together as a residual block is trained, against 64-bit autograd; then
    recorded into a graph whose replays, with eager calls on the same contexts between
    them, give the eager bits for the state they find."""
    g = torch.Generator().manual_seed(rows)
    W1, b1 = _layer(g, d, f, dtype, True)
    W2, b2 = _layer(g, f, d, dtype, True)
    _, x = _rows(g, rows, d, dtype, 0)
    _, dy = _rows(g, rows, d, dtype, 0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        rng = _rng(21, 5)
        ctx1 = mlp.mlp_linear_init(W1, b1, "gelu", max_rows=rows)
        ctx2 = mlp.mlp_linear_init(W2, b2, "none", max_rows=rows)
        got = _block_loss(mlp, ctx1, ctx2, x, dy, rng)
        torch.cuda.synchronize()
        ps = [t.cpu().double().requires_grad_() for t in (x, W1, b1, W2, b2)]
        h = R.act(ps[0] @ ps[1] + ps[2], "gelu")
        y = ps[0] + (h @ ps[3] + ps[4]) * R.factor((21, 5), rows, d, 0.1)
        y.backward(dy.cpu().double())
        # normwise: each of at most four roundings to the type on the way (h, z, dh, g)
        # and the result's, u each at most, and the products' own sums
        bar = 6 * R.U[dtype] + 64 * R.E
        for name, a, b in zip(("y", "dx", "dW1", "db1", "dW2", "db2"), got, [y] + [t.grad for t in ps]):
            e = float((a.cpu().double() - b.detach()).norm() / b.detach().norm())
            print("%-4s %.2e (bar %.1e)" % (name, e, bar), flush=True)
            assert e <= bar, name
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=s):
            held = _block_loss(mlp, ctx1, ctx2, x, dy, rng)
        for k in range(4):
            gr.replay()
            torch.cuda.synchronize()
            replayed = [t.clone() for t in held]
            eager = _block_loss(mlp, ctx1, ctx2, x, dy, rng)
            torch.cuda.synchronize()
            for a, b in zip(replayed, eager):
                assert torch.equal(a, b)
            rng[1] += 1000
            x.mul_(-0.5)
            torch.cuda.synchronize()


def test_own_stream(mlp):  # noqa: F811
    """A context with a stream of its own, called while another stream is current."""
    g = torch.Generator().manual_seed(6)
    W, b = _layer(g, 128, 256, "bf16", True)
    _, x = _rows(g, 500, 128, "bf16", 0)
    _, dy = _rows(g, 500, 256, "bf16", 0)
    plain = mlp.mlp_linear_init(W, b, "silu", max_rows=500)
    want = mlp.mlp_linear_forward(plain, x, save_z=True)
    wantg = mlp.mlp_linear_backward(plain, x, dy, z=want[1])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    ctx = mlp.mlp_linear_init(W, b, "silu", max_rows=500, stream=s.cuda_stream)
    for _ in range(3):
        got = mlp.mlp_linear_forward(ctx, x, save_z=True)
        gotg = mlp.mlp_linear_backward(ctx, x, dy, z=got[1])
        s.synchronize()
        for a, c in zip(got + gotg, want + wantg):
            assert torch.equal(a, c)
    mlp.mlp_linear_set_stream(ctx, None)
    assert torch.equal(mlp.mlp_linear_forward(ctx, x), want[0])


def test_calls_follow_one_another_over_streams(mlp):  # noqa: F811
    """A context without a stream of its own, made on one stream and called on others: a
    call comes after the ones before it, whose workspace it shares (the split sums and
    arrival counts of few rows, g of the backward call)."""
    g = torch.Generator().manual_seed(7)
    W, b = _layer(g, 4096, 256, "bf16", True)
    _, x = _rows(g, 6, 4096, "bf16", 0)
    _, dy = _rows(g, 6, 256, "bf16", 0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    with torch.cuda.stream(streams[0]):
        ctx = mlp.mlp_linear_init(W, b, "silu", max_rows=6)
    state, out = _rng(1, 2), []
    torch.cuda.synchronize()
    for i in range(12):
        with torch.cuda.stream(streams[i % 3]):
            y, z = mlp.mlp_linear_forward(ctx, x, save_z=True)
            out.append((y, z) + mlp.mlp_linear_backward(ctx, x, dy, z=z, p=0.5, rng=state))
    torch.cuda.synchronize()
    ry, rz, by, bz = R.forward(x, W, b, None, "silu", 0.0, None, "bf16")
    R.check("y", out[0][0], ry, by)
    R.check("z", out[0][1], rz, bz)
    for o in out[1:]:
        assert all(torch.equal(a, c) for a, c in zip(o, out[0]))


def test_two_contexts_at_once(mlp):  # noqa: F811
    """Two layers with workspaces of their own, on two streams at the same time."""
    g = torch.Generator().manual_seed(8)
    jobs = []
    for rows, d_in, d_out in ((5, 4096, 384), (700, 520, 264)):
        W, b = _layer(g, d_in, d_out, "bf16", True)
        _, x = _rows(g, rows, d_in, "bf16", 0)
        s = torch.cuda.Stream()
        ctx = mlp.mlp_linear_init(W, b, "relu", max_rows=rows, stream=s.cuda_stream)
        want = R.forward(x, W, b, None, "relu", 0.0, None, "bf16")
        jobs.append((ctx, x, s, want))
    torch.cuda.synchronize()
    got = [[mlp.mlp_linear_forward(ctx, x) for ctx, x, _, _ in jobs] for _ in range(20)]
    torch.cuda.synchronize()
    for j, (_, _, _, want) in enumerate(jobs):
        R.check("y", got[0][j], want[0], want[2])
        assert all(torch.equal(o[j], got[0][j]) for o in got)


def test_few_rows_in_a_graph(mlp):  # noqa: F811
    """Split sums and their arrival counts over replays, with eager calls in between."""
    g = torch.Generator().manual_seed(9)
    W, b = _layer(g, 4096, 384, "bf16", True)
    _, x = _rows(g, 3, 4096, "bf16", 0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ctx = mlp.mlp_linear_init(W, b, "gelu_tanh", max_rows=20)
        y = mlp.mlp_linear_forward(ctx, x)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=s):
            mlp.mlp_linear_forward(ctx, x, out=y)
        for k in range(5):
            gr.replay()
            gr.replay()
            torch.cuda.synchronize()
            replayed = y.clone()
            assert torch.equal(mlp.mlp_linear_forward(ctx, x), replayed)
            ry, _, by, _ = R.forward(x, W, b, None, "gelu_tanh", 0.0, None, "bf16")
            R.check("y", replayed, ry, by)
            x.mul_(-0.75)
            torch.cuda.synchronize()


def test_refusals(mlp):  # noqa: F811
    W = torch.zeros(16, 24, device="cuda")
    b = torch.zeros(24, device="cuda")
    ctx = mlp.mlp_linear_init(W, b, "relu", max_rows=8)
    x, y = torch.zeros(8, 16, device="cuda"), torch.full((8, 24), 5.0, device="cuda")
    z, r = torch.zeros(8, 24, device="cuda"), _rng(1, 2)
    with pytest.raises(mlp.MLPError):
        mlp.mlp_linear_forward(ctx, torch.zeros(9, 16, device="cuda"))
    for p in (-0.5, 1.5, float("nan")):
        with pytest.raises(mlp.MLPError):
            mlp.mlp_linear_forward(ctx, x, p=p, rng=r, out=y)
        with pytest.raises(mlp.MLPError):
            mlp.mlp_linear_backward(ctx, x, y, z=z, p=p, rng=r)
    with pytest.raises(mlp.MLPError):
        mlp.mlp_linear_forward(ctx, x, p=0.5, out=y)
    with pytest.raises(mlp.MLPError):
        mlp.mlp_linear_forward(ctx, x, out=y, z=y)
    with pytest.raises(mlp.MLPError):
        mlp.mlp_linear_backward(ctx, x, y)                   # no z
    with pytest.raises(mlp.MLPError):
        mlp.mlp_linear_backward(ctx, None, y, z=z)           # dW without X
    with pytest.raises(mlp.MLPError):
        mlp.mlp_linear_backward(ctx, x, y, z=z, dX=x)
    with pytest.raises(mlp.MLPError):
        mlp.mlp_linear_backward(ctx, x, y, z=z, dW=W)
    for bad in (x.bfloat16(), x.cpu(), x.double()):
        with pytest.raises(TypeError):
            mlp.mlp_linear_forward(ctx, bad, out=y)
    for bad in (x[:, :8], x.t().contiguous().t(), x[:1].expand(8, 16)):
        with pytest.raises(ValueError):
            mlp.mlp_linear_forward(ctx, bad, out=y)
    with pytest.raises(ValueError):
        mlp.mlp_linear_init(W, b[:8], "relu", max_rows=8)
    with pytest.raises(ValueError):
        mlp.mlp_linear_init(W, b, "relu", max_rows=8, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(KeyError):
        mlp.mlp_linear_init(W, b, "swish", max_rows=8)
    with pytest.raises(TypeError):
        mlp.mlp_linear_init(W.double(), None, "relu", max_rows=8)
    torch.cuda.synchronize()
    assert bool((y == 5.0).all())


@pytest.mark.parametrize("act", R.ACTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_activations_far_out(mlp, dtype, act):  # noqa: F811
    """a(z) and a'(z) where powers of z leave fp32: of one row through the unit matrix."""
    big = [0.0, 3.0, 20.0, 100.0, 1e4, 6e4] + ([] if dtype == "f16" else [1e19, 1e20, 3e38])
    z = torch.tensor([[s * v for v in big for s in (1, -1)]]).to(R.DTYPES[dtype]).cuda()
    n = z.shape[1]
    ctx = mlp.mlp_linear_init(torch.eye(n, device="cuda", dtype=z.dtype), torch.zeros_like(z[0]), act, max_rows=1)
    y = mlp.mlp_linear_forward(ctx, z)
    _, _, db = mlp.mlp_linear_backward(ctx, None, torch.ones_like(z), z=z, need_dx=False, need_dw=False)
    u, zd = R.U[dtype], z.cpu().double()
    # the functions to a few 2^-24 of their terms, |z| of them no more than where they have
    # not reached their ends (20), and the rounding of the result
    for got, want, size in ((y, R.act(zd, act), zd.abs()), (db[None], R.act_grad(zd, act), zd.abs().clamp(max=20))):
        R.check(act, got, want, u * want.abs() + 16 * R.E * (1 + size) + R.TINY[dtype])


@pytest.mark.parametrize("rows", [0, 4])
def test_outputs_that_are_parameters(mlp, rows):  # noqa: F811
    """No call takes W or the bias as an output, not of no rows either."""
    W = torch.ones(16, 16, device="cuda")
    b = torch.ones(16, device="cuda")
    ctx = mlp.mlp_linear_init(W, b, max_rows=4)
    x = torch.ones(rows, 16, device="cuda")
    for bad in (dict(dW=W), dict(db=b)):
        with pytest.raises(mlp.MLPError):
            mlp.mlp_linear_backward(ctx, x, torch.ones_like(x), **bad)
    torch.cuda.synchronize()
    assert bool((W == 1).all()) and bool((b == 1).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d_out", range(1, 8))
def test_narrow_and_deep(mlp, dtype, d_out):  # noqa: F811
    """Fewer than eight outputs of a deep row: every width, rows and depths around a step."""
    for i, (rows, d_in) in enumerate([(1, 511), (3, 512), (9, 1024), (8, 4096), (17, 4099), (33, 8191), (1101, 2050)]):
        act, p, bias, residual, _ = OPTIONS[(i + d_out) % 5]
        print(dtype, rows, d_in, d_out, act, p, bias, residual, flush=True)
        g = torch.Generator().manual_seed(i)
        W, b = _layer(g, d_in, d_out, dtype, bias)
        _, x = _rows(g, rows, d_in, dtype, i, float("nan"))
        r = _rows(g, rows, d_out, dtype, i, float("nan"))[1] if residual else None
        ybuf, y = _rows(g, rows, d_out, dtype, 2)
        zbuf, z = _rows(g, rows, d_out, dtype, 1)
        ctx = mlp.mlp_linear_init(W, b, act, max_rows=rows)
        mlp.mlp_linear_forward(ctx, x, residual=r, p=p, rng=_rng(5, i), out=y, z=z)
        torch.cuda.synchronize()
        ry, rz, by, bz = R.forward(x, W, b, r, act, p, (5, i), dtype)
        R.check("y", y, ry, by)
        R.check("z", z, rz, bz)
        assert bool((ybuf[:, d_out:] == 7.0).all()) and bool((zbuf[:, d_out:] == 7.0).all())


# either side of the rules between few rows and tiles, of splits and of deep thin products
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,d_in,d_out", [(300, 40, 5001), (100, 200, 6000), (200, 5000, 24), (600, 4104, 129),
                                             (520, 776, 520), (48, 4099, 520), (2050, 72, 200), (4100, 260, 136)])
def test_between_the_rules(mlp, dtype, rows, d_in, d_out):  # noqa: F811
    print(dtype, rows, d_in, d_out, flush=True)
    g = torch.Generator().manual_seed(rows)
    W, b = _layer(g, d_in, d_out, dtype, True)
    _, x = _rows(g, rows, d_in, dtype, 0)
    _, dy = _rows(g, rows, d_out, dtype, 1)
    ctx = mlp.mlp_linear_init(W, b, "silu", max_rows=rows)
    y, z = mlp.mlp_linear_forward(ctx, x, p=0.1, rng=_rng(3, 4), save_z=True)
    dx, dw, db = mlp.mlp_linear_backward(ctx, x, dy, z=z, p=0.1, rng=_rng(3, 4))
    plain = mlp.mlp_linear_init(W, None, "none", max_rows=rows)
    px, pw, _ = mlp.mlp_linear_backward(plain, x, dy)
    torch.cuda.synchronize()
    ry, rz, by, bz = R.forward(x, W, b, None, "silu", 0.1, (3, 4), dtype)
    R.check("y", y, ry, by)
    R.check("z", z, rz, bz)
    for got, (ref, bound) in (((dx, dw, db), R.backward(x, W, z, dy, "silu", 0.1, (3, 4), dtype)),
                              ((px, pw, None), R.backward(x, W, None, dy, "none", 0.0, None, dtype))):
        for name, t in zip(("dx", "dw", "db"), got):
            if t is not None:
                R.check(name, t, ref[name], bound[name])
