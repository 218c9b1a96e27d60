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
