"""The workspace of a dense layer's context between streams: its memory is not handed out
while a call uses it, nor taken from under pending work of another stream."""
import pytest
import torch

from tests import layers_ref as R
from tests.test_gpu_dropout import _rows, mlp  # noqa: F401
from tests.test_gpu_linear import _layer

pytestmark = pytest.mark.gpu


def _busy(a):
    """About 20 ms of work on the current stream."""
    for _ in range(20):
        a = a @ a * 1e-3
    return a


def _problem():
    g = torch.Generator().manual_seed(1)
    W, b = _layer(g, 4096, 384, "bf16", True)
    return W, b, _rows(g, 5, 4096, "bf16", 0)[1]


def test_dropped_while_a_call_is_under_way(mlp):  # noqa: F811
    W, b, x = _problem()
    a = torch.randn(8192, 8192, device="cuda")
    _busy(a)
    ctx = mlp.mlp_linear_init(W, b, "silu", max_rows=5)
    at, n = ctx.workspace.data_ptr(), ctx.workspace.numel()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        held = _busy(a)
        y = mlp.mlp_linear_forward(ctx, x)
    del ctx                                     # the call has not started
    taken = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(3)]
    assert not side.query(), "the side stream was done too soon for this test"
    assert all(t.data_ptr() != at for t in taken)
    for t in taken:
        t.fill_(0x5A)
    torch.cuda.synchronize()
    ry, _, by, _ = R.forward(x, W, b, None, "silu", 0.0, None, "bf16")
    R.check("y", y, ry, by)
    assert all(bool((t == 0x5A).all()) for t in taken) and held.shape == a.shape


@pytest.mark.parametrize("default", [False, True])
def test_made_on_a_stream_of_its_own_while_another_is_busy(mlp, default):  # noqa: F811
    W, b, x = _problem()
    a = torch.randn(8192, 8192, device="cuda")
    n = mlp.mlp_linear_workspace_bytes(W.dtype, 4096, 384, 5)
    own, busy = torch.cuda.default_stream() if default else torch.cuda.Stream(), torch.cuda.Stream()
    _busy(a)
    torch.cuda.synchronize()
    with torch.cuda.stream(busy):
        t = torch.empty(n, dtype=torch.uint8, device="cuda")
        at = t.data_ptr()
        held = _busy(a)
        t.fill_(0x5A)                           # pending; its block is free for this stream
        del t
        ctx = mlp.mlp_linear_init(W, b, "silu", max_rows=5, stream=own.cuda_stream)
        assert ctx.workspace.data_ptr() != at
        ys = [mlp.mlp_linear_forward(ctx, x) for _ in range(3)]
    torch.cuda.synchronize()
    ry, _, by, _ = R.forward(x, W, b, None, "silu", 0.0, None, "bf16")
    for y in ys:
        R.check("y", y, ry, by)
    assert held.shape == a.shape


def test_layers_that_share_a_workspace(mlp):  # noqa: F811
    """Layers of other shapes and types, one after the other on one workspace: the arrival
    counts that one leaves zero are not where another keeps its sums."""
    jobs, need = [], 0
    shapes = [("bf16", 4, 4096, 384), ("f32", 6, 2048, 520), ("f16", 300, 264, 1001), ("bf16", 64, 1032, 7), ("f32", 700, 96, 40)]
    for i, (dtype, rows, d_in, d_out) in enumerate(shapes):
        g = torch.Generator().manual_seed(i)
        W, b = _layer(g, d_in, d_out, dtype, True)
        _, x = _rows(g, rows, d_in, dtype, 0)
        _, dy = _rows(g, rows, d_out, dtype, 0)
        need = max(need, mlp.mlp_linear_workspace_bytes(W.dtype, d_in, d_out, rows))
        jobs.append((W, b, x, dy))

    def call(ctx, x, dy):
        y, z = mlp.mlp_linear_forward(ctx, x, save_z=True)
        return (y, z) + mlp.mlp_linear_backward(ctx, x, dy, z=z)

    own = [call(mlp.mlp_linear_init(W, b, "gelu", max_rows=x.shape[0]), x, dy) for W, b, x, dy in jobs]
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    ctxs = [mlp.mlp_linear_init(W, b, "gelu", max_rows=x.shape[0], workspace=work) for W, b, x, _ in jobs]
    for _ in range(3):
        got = [call(c, x, dy) for c, (_, _, x, dy) in zip(ctxs, jobs)]
        torch.cuda.synchronize()
        for a, w in zip(got, own):
            assert all(torch.equal(s, t) for s, t in zip(a, w))


def test_without_max_rows(mlp):  # noqa: F811
    """A context takes memory for the rows it is called with (2^20 rows of this layer: 8 GiB),
    and calls of any rows work; captured ones replay after the workspace has grown."""
    g = torch.Generator().manual_seed(3)
    W, b = _layer(g, 1000, 1001, "bf16", True)
    _, x = _rows(g, 3000, 1000, "bf16", 0)
    _, dy = _rows(g, 3000, 1001, "bf16", 0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda.synchronize()
        taken = torch.cuda.memory_allocated()
        ctx = mlp.mlp_linear_init(W, b, "silu")
        assert torch.cuda.memory_allocated() - taken < 64 << 20
        big = mlp.mlp_linear_init(W, b, "silu", max_rows=3000)
        small = x[:500].clone()
        want = mlp.mlp_linear_forward(big, small)
        out = mlp.mlp_linear_forward(ctx, small)
        torch.cuda.synchronize()
        gr, too_many = torch.cuda.CUDAGraph(), torch.empty(3000, 1001, dtype=W.dtype, device="cuda")
        with torch.cuda.graph(gr, stream=s):
            mlp.mlp_linear_forward(ctx, small, out=out)
            with pytest.raises(mlp.MLPError):       # no room, and none is made in a capture
                mlp.mlp_linear_forward(ctx, x, out=too_many)
        for rows in (1024, 1025, 3000):
            z = mlp.mlp_linear_forward(big, x[:rows], save_z=True)
            assert all(torch.equal(a, c) for a, c in zip(mlp.mlp_linear_forward(ctx, x[:rows], save_z=True), z))
            for a, c in zip(mlp.mlp_linear_backward(ctx, x[:rows], dy[:rows], z=z[1]),
                            mlp.mlp_linear_backward(big, x[:rows], dy[:rows], z=z[1])):
                assert torch.equal(a, c)
            out.zero_()
            gr.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
        assert ctx.max_rows == 4096 and len(ctx.before) == 2
    with pytest.raises(mlp.MLPError):
        mlp.mlp_linear_forward(big, torch.empty(3001, 1000, dtype=W.dtype, device="cuda"))


@pytest.mark.parametrize("rows", [3, 300])
def test_captured_on_a_stream_of_the_graphs_own(mlp, rows):  # noqa: F811
    """Eager calls on one stream, a capture on the stream that torch makes for it, replays with
    eager calls of other rows in between, the context dropped after the last."""
    g = torch.Generator().manual_seed(rows)
    W, b = _layer(g, 2048, 264, "bf16", True)
    _, x = _rows(g, rows, 2048, "bf16", 0)
    _, dy = _rows(g, rows, 264, "bf16", 0)
    ctx = mlp.mlp_linear_init(W, b, "gelu")

    def call(k):
        y, z = mlp.mlp_linear_forward(ctx, x[:k], save_z=True)
        return (y, z) + mlp.mlp_linear_backward(ctx, x[:k], dy[:k], z=z)

    call(rows)
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        held = call(rows)
    side = torch.cuda.Stream()
    for k in range(4):
        gr.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in held]
        with torch.cuda.stream(side):
            call(rows - 1)
        eager = call(rows)
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(replayed, eager))
        x.mul_(-0.5)
        torch.cuda.synchronize()
    gr.reset()
    del ctx
    torch.cuda.synchronize()
