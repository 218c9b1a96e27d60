"""Host-side checks of the layer calls that need no GPU: sizes and refusals (the pointers
are never dereferenced)."""
import ctypes

from tests.test_abi_host import _lib

F = ctypes.c_void_p(4096)
G = ctypes.c_void_p(8192)
H = ctypes.c_void_p(12288)
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3


def test_workspace_bytes():
    lib = _lib()
    for dtype in (0, 1, 2):
        for d_in, d_out, rows in ((1, 1, 1), (32, 256, 4096), (4096, 4096, 8192), (1 << 20, 1, 1), (1, 1 << 20, 3)):
            b = lib.mlp_linear_workspace_bytes(dtype, d_in, d_out, rows)
            assert b > 0 and b % 256 == 0
            assert lib.mlp_linear_workspace_bytes(dtype, d_in, d_out, rows + 500) >= b
    for bad in ((3, 8, 8, 8), (-1, 8, 8, 8), (0, 0, 8, 8), (0, 8, 0, 8), (0, 8, 8, 0), (0, -5, 8, 8),
                (0, (1 << 20) + 1, 8, 8), (0, 8, (1 << 20) + 1, 8), (0, 8, 8, (1 << 20) + 1)):
        assert lib.mlp_linear_workspace_bytes(*bad) == 0


def test_init_refuses():
    lib = _lib()
    h = ctypes.c_void_p()
    ws = lib.mlp_linear_workspace_bytes(1, 64, 64, 64)

    def init(out=ctypes.byref(h), dtype=1, d_in=64, d_out=64, act=1, rows=64, w=F, work=G, n=ws):
        return lib.mlp_linear_init(out, dtype, d_in, d_out, act, rows, w, None, work, n, None)

    assert init(out=None) == INVALID and init(w=None) == INVALID and init(work=None) == INVALID
    assert init(dtype=3) == UNSUPPORTED and init(d_in=0) == UNSUPPORTED and init(rows=0) == UNSUPPORTED
    assert init(act=5) == UNSUPPORTED and init(act=-1) == UNSUPPORTED
    assert init(n=ws - 1) == WORKSPACE and init(work=ctypes.c_void_p(8192 + 16)) == WORKSPACE
    assert h.value is None


def test_null_context():
    lib = _lib()
    assert lib.mlp_linear_forward(None, F, 8, 1, None, 0, 0.0, None, G, 8, None, 0) == INVALID
    assert lib.mlp_linear_backward(None, F, 8, None, 0, G, 8, 1, 0.0, None, H, 8, None, None) == INVALID
    assert lib.mlp_linear_set_stream(None, None) == INVALID
    lib.mlp_linear_destroy(None)


def test_dropout_refuses():
    lib = _lib()

    def fwd(dtype=0, rows=4, cols=8, x=F, ldx=8, r=None, ldr=0, p=0.5, rng=H, y=G, ldy=8):
        return lib.mlp_dropout_forward(dtype, rows, cols, x, ldx, r, ldr, p, rng, y, ldy, None)

    def bwd(dtype=0, rows=4, cols=8, x=F, ldx=8, p=0.5, rng=H, y=G, ldy=8):
        return lib.mlp_dropout_backward(dtype, rows, cols, x, ldx, p, rng, y, ldy, None)

    for call in (fwd, bwd):
        assert call(dtype=3) == UNSUPPORTED and call(dtype=-1) == UNSUPPORTED
        assert call(rows=-1) == INVALID and call(cols=-1) == INVALID
        for p in (-0.01, 1.01, float("nan"), float("inf"), float("-inf")):
            assert call(p=p) == INVALID
        assert call(rng=None) == INVALID
        assert call(x=None) == INVALID and call(y=None) == INVALID
        assert call(ldx=7) == INVALID and call(ldy=7) == INVALID
        assert call(ldx=1 << 45) == INVALID and call(ldy=1 << 45) == INVALID
        assert call(rows=1 << 40, cols=1 << 40) == INVALID
        assert call(y=F, ldy=9) == INVALID                       # X at another stride
        assert call(rows=0, x=None, y=None) == 0 and call(cols=0, x=None, y=None) == 0
        assert call(rows=0, p=2.0) == INVALID
    assert fwd(r=H, ldr=7) == INVALID and fwd(r=G, ldr=9) == INVALID
