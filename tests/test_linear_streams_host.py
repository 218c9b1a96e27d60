"""Which streams the binding of the dense layer allocates on, waits for and reports to the
allocator, on stand-ins for torch's streams and memory (no GPU)."""
import contextlib
import types

import pytest
import torch

from paper_2606_30497_amd import mlp


class Stream:
    def __init__(self, world, handle):
        self.world, self.cuda_stream = world, handle

    def wait_stream(self, other):
        self.world.log.append(("wait", self.cuda_stream, other.cuda_stream))


class Memory:
    """What torch.empty gives: the stream whose pool it is from, and those it was told of."""

    def __init__(self, world, shape, dtype=torch.float32):
        self.world, self.shape, self.dtype = world, shape, dtype
        self.device, self.pool, self.recorded = types.SimpleNamespace(index=0), world.current, set()

    def dim(self):
        return len(self.shape)

    def numel(self):
        return 1 << 20

    def data_ptr(self):
        return 4096

    def record_stream(self, s):
        self.recorded.add(s.cuda_stream)


class World:
    """torch.cuda of one device: 0 is its default stream, a stream made of the handle 0 is a
    new one (as torch's are), `capturing` the handles of streams that capture."""

    def __init__(self):
        self.current, self.capturing, self.log = 0, set(), []
        self.device = lambda device: contextlib.nullcontext()

    def ExternalStream(self, handle, device=None):
        return Stream(self, handle or 9999)

    def default_stream(self, device=None):
        return Stream(self, 0)

    def current_stream(self, device=None):
        return Stream(self, self.current)

    def is_current_stream_capturing(self):
        return self.current in self.capturing

    @contextlib.contextmanager
    def stream(self, s):
        before, self.current = self.current, s.cuda_stream
        yield
        self.current = before


class Lib:
    """The library: where its context is."""

    def __init__(self, world):
        self.world, self.on = world, None

    def mlp_linear_workspace_bytes(self, *a):
        return 4096

    def mlp_linear_init(self, *a):
        self.on = a[-1]
        self.world.log.append(("clear", a[-1]))
        return 0

    def mlp_linear_set_stream(self, handle, stream):
        self.on = stream
        return 0


@pytest.fixture
def world(monkeypatch):
    w = World()
    lib = Lib(w)
    w.lib = lib
    fake = types.SimpleNamespace(cuda=w, uint8=torch.uint8, Tensor=torch.Tensor,
                                 empty=lambda shape, dtype, device: Memory(w, shape, dtype))
    monkeypatch.setattr(mlp, "torch", fake)
    monkeypatch.setattr(mlp, "load", lambda: lib)
    monkeypatch.setattr(mlp, "_lib", None)
    monkeypatch.setattr(mlp, "_dev", lambda t, *a, **k: t.data_ptr())
    monkeypatch.setattr(mlp, "_current_stream", lambda index: w.current)
    return w


def _layer(world, **k):
    return mlp.mlp_linear_init(Memory(world, (16, 24)), None, "none", max_rows=8, **k)


def test_the_default_stream_given_by_its_handle(world):
    """Outputs of a context on the stream 0 are from the default stream's pool."""
    ctx = _layer(world, stream=0)
    world.current = 5
    assert mlp._new(ctx, 8, 24).pool == 0


def test_workspace_is_from_the_pool_of_the_stream_that_clears_it(world):
    """What is pending on the current stream may still write to the block that its pool gives:
    the clear of the arrival counts on another stream would not come after it."""
    world.current = 5
    for given, pool in ((None, 5), (7, 7), (0, 0)):
        ctx = _layer(world, stream=given)
        assert ctx.workspace.pool == pool and world.log[-1] == ("clear", pool)


def test_allocator_knows_the_streams_of_the_workspace(world):
    """A context made on one stream and called on others gives its workspace back to the
    first one's pool: only what the allocator was told of keeps it from the next tensor."""
    world.current = 5
    ctx = _layer(world)
    for s in (5, 6, 5, 0):
        world.current = s
        mlp._bind_stream(ctx)
        assert world.lib.on == s
    mlp.mlp_linear_set_stream(ctx, 8)
    assert ctx.workspace.recorded | {5} == {5, 6, 0, 8}
    own = _layer(world, stream=7)
    mlp.mlp_linear_set_stream(own, None)
    world.current = 6
    mlp._bind_stream(own)
    assert own.workspace.recorded | {7} == {7, 6}


def test_calls_wait_for_those_before_them(world):
    """Each call that is not captured waits for the last one that was not, whose workspace it
    shares; a capture on another stream in between changes nothing in that."""
    world.current = 5
    ctx = _layer(world)
    del world.log[:]

    def call(stream, *waits):
        world.current = stream
        mlp._bind_stream(ctx)
        assert world.lib.on == stream and world.log == list(waits), (stream, world.log)
        del world.log[:]

    call(5)
    call(6, ("wait", 6, 5))
    call(6)
    world.capturing = {7}
    call(7)                       # recorded, not run: nothing to wait for or to be waited for
    call(7)
    call(8, ("wait", 8, 6))       # while 7 still captures: an event of 7 would draw 8 into the capture
    call(7)
    world.capturing = set()
    call(7, ("wait", 7, 8))       # the library's context is on 7 already
    call(0, ("wait", 0, 7))
    mlp.mlp_linear_set_stream(ctx, 9)
    assert world.log == [("wait", 9, 0)] and world.lib.on == 9
    del world.log[:]
    world.current = 5
    mlp._bind_stream(ctx)         # a stream of its own: the current one does not matter
    assert world.log == [] and world.lib.on == 9
    mlp.mlp_linear_set_stream(ctx, None)
    call(5, ("wait", 5, 9))


def test_workspaces_of_the_whole_nets(world):
    """The same for mlp_init, mlp_set_strategy and mlp_deep_init, whose calls all go on the
    context's own stream."""
    lib, world.current = world.lib, 5
    for name in ("mlp_workspace_bytes", "mlp_strategy_workspace_bytes", "mlp_deep_workspace_bytes", "mlp_deep_param_count"):
        setattr(lib, name, lambda *a: 4096)
    for name in ("mlp_init", "mlp_set_stream", "mlp_set_strategy", "mlp_deep_init"):
        setattr(lib, name, lambda *a: 0)
    w = Memory(world, (32, 64))
    for given, pool in ((None, 5), (7, 7), (0, 0)):
        ctx = mlp.mlp_init(w, w, 64, stream=given)
        mlp.mlp_set_strategy(ctx, "tile")
        assert ctx.workspace.pool == ctx.strategy_workspace.pool == pool
        assert mlp.mlp_deep_init(w, 64, 2, 64, stream=given).workspace.pool == pool
        mlp.mlp_set_stream(ctx, 8)
        assert ctx.workspace.recorded == ctx.strategy_workspace.recorded == {8}
        mlp.mlp_set_strategy(ctx, "baseline")
        assert ctx.strategy_workspace.pool == 8


def test_a_context_that_grows(world):
    """On the stream of its calls; what the library refuses is left to it."""
    made = []
    world.lib.mlp_linear_init = lambda *a: made.append((a[5], a[-1])) or 0
    world.lib.mlp_linear_destroy = lambda h: None
    world.current = 5
    ctx = mlp.mlp_linear_init(Memory(world, (16, 24)), None, "none")
    first = ctx.workspace
    assert ctx.grows and made == [(1024, 5)]
    world.current = 6
    mlp._bind_stream(ctx)
    mlp._grow(ctx, 1025)
    assert made[1:] == [(2048, 6)] and ctx.workspace.pool == 6 and ctx.max_rows == 2048 and ctx.before == [first]
    world.capturing = {6}
    mlp._grow(ctx, 5000)
    world.capturing = set()
    mlp._grow(ctx, mlp.MAX_BATCH + 1)
    assert len(made) == 2
    mlp._grow(ctx, mlp.MAX_BATCH)
    assert made[2:] == [(mlp.MAX_BATCH, 6)]
    assert not _layer(world).grows
