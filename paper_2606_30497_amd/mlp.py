"""Thin ctypes binding of libmlp.so (include/mlp.h).

Argument marshalling only: every step of the training path runs in the HIP
kernels of libmlp.so. torch supplies device memory and the stream; tensors are
checked for device, dtype, shape and contiguity, then their data pointers are
passed through. There is no CPU fallback: if the library or a GPU is missing,
every call raises.
"""
from __future__ import annotations

import ctypes
import os

import torch

from . import build as _build

D_IN = 32
HIDDEN_SIZES = (32, 64, 128, 256, 512, 1024)
MAX_BATCH = 1 << 20

MLP_OK = 0
STATUS = {0: "MLP_OK", -1: "MLP_ERR_INVALID_ARG", -2: "MLP_ERR_UNSUPPORTED",
          -3: "MLP_ERR_WORKSPACE", -4: "MLP_ERR_HIP", -5: "MLP_ERR_NONFINITE",
          -6: "MLP_ERR_INDEX", -7: "MLP_ERR_TIMEOUT"}

STRATEGY_FUSED, STRATEGY_TILE, STRATEGY_OPTIMIZED, STRATEGY_BASELINE = 0, 1, 2, 3
STRATEGIES = {"fused": STRATEGY_FUSED, "tile": STRATEGY_TILE, "optimized": STRATEGY_OPTIMIZED,
              "baseline": STRATEGY_BASELINE}

EXPORTS = ("mlp_workspace_bytes", "mlp_init", "mlp_set_stream", "mlp_strategy_workspace_bytes",
           "mlp_set_strategy", "mlp_forward", "mlp_backward",
           "mlp_sgd_step", "mlp_train_epochs", "mlp_check_errors", "mlp_profile",
           "mlp_last_kernel_ms", "mlp_launch_info", "mlp_phase_cycles", "mlp_destroy",
           "mlp_train_epochs_static", "mlp_status_string",
           "mlp_deep_param_count", "mlp_deep_workspace_bytes", "mlp_deep_init", "mlp_deep_forward",
           "mlp_deep_backward", "mlp_deep_sgd_step", "mlp_deep_train_epochs",
           "mlp_deep_check_errors", "mlp_deep_profile", "mlp_deep_last_kernel_ms",
           "mlp_deep_destroy",
           "mlp_linear_workspace_bytes", "mlp_linear_init", "mlp_linear_set_stream",
           "mlp_linear_forward", "mlp_linear_backward", "mlp_linear_destroy",
           "mlp_dropout_forward", "mlp_dropout_backward")


class MLPError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (fn, STATUS.get(status, "?"), status))


_lib = None

_vp = ctypes.c_void_p
_i32 = ctypes.c_int32
_i64 = ctypes.c_int64
_f32 = ctypes.c_float


def library_path() -> str:
    """The in-tree libmlp.so, or another build of it that MLP_LIBRARY names."""
    return os.environ.get("MLP_LIBRARY") or _build.LIB


def load(require_built: bool = True):
    """Load libmlp.so (after torch, so that both share one HIP runtime)."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        if require_built or path != _build.LIB:
            raise RuntimeError("%s is not built (run __graft_entry__.build())" % path)
        _build.build()
    lib = ctypes.CDLL(path)
    sig = {
        "mlp_workspace_bytes": (ctypes.c_size_t, [_i32, _i32, _i64]),
        "mlp_init": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i32, _i32, _i64, _vp, _vp, _vp,
                                    ctypes.c_size_t, _vp]),
        "mlp_set_stream": (ctypes.c_int, [_vp, _vp]),
        "mlp_strategy_workspace_bytes": (ctypes.c_size_t, [_i32, _i32, _i64, _i32]),
        "mlp_set_strategy": (ctypes.c_int, [_vp, _i32, _vp, ctypes.c_size_t]),
        "mlp_forward": (ctypes.c_int, [_vp, _vp, _i64, _vp, _i64, _vp]),
        "mlp_backward": (ctypes.c_int, [_vp, _vp, _i64, _vp, _vp, _i64, _vp, _vp, _vp]),
        "mlp_sgd_step": (ctypes.c_int, [_vp, _vp, _i64, _vp, _vp, _i64, _f32, _vp]),
        "mlp_train_epochs": (ctypes.c_int, [_vp, _vp, _vp, _i64, _i64, _f32, _i32, _vp, _i64,
                                            _vp, _vp]),
        "mlp_check_errors": (ctypes.c_int, [_vp]),
        "mlp_profile": (ctypes.c_int, [_vp, _i32]),
        "mlp_last_kernel_ms": (ctypes.c_int, [_vp, ctypes.POINTER(_f32)]),
        "mlp_launch_info": (ctypes.c_int, [_vp, _i64, _i64, _i32, ctypes.POINTER(_i32),
                                           ctypes.POINTER(_i64)]),
        "mlp_phase_cycles": (ctypes.c_int, [_vp, _vp, _i64, ctypes.POINTER(_i64)]),
        "mlp_train_epochs_static": (ctypes.c_int, [_i32, _vp, _vp, _vp, _vp, _i64, _i64, _f32, _i32,
                                                   _vp, _i64, _vp, _vp, _vp, _vp]),
        "mlp_destroy": (None, [_vp]),
        "mlp_status_string": (ctypes.c_char_p, [ctypes.c_int]),
        "mlp_deep_param_count": (_i64, [_i32, _i32, _i32]),
        "mlp_deep_workspace_bytes": (ctypes.c_size_t, [_i32, _i32, _i32, _i64]),
        "mlp_deep_init": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i32, _i32, _i32, _i64, _vp,
                                         _vp, ctypes.c_size_t, _vp]),
        "mlp_deep_forward": (ctypes.c_int, [_vp, _vp, _i64, _vp, _i64, _vp]),
        "mlp_deep_backward": (ctypes.c_int, [_vp, _vp, _i64, _vp, _vp, _i64, _vp, _vp]),
        "mlp_deep_sgd_step": (ctypes.c_int, [_vp, _vp, _i64, _vp, _vp, _i64, _f32, _vp]),
        "mlp_deep_train_epochs": (ctypes.c_int, [_vp, _vp, _vp, _i64, _i64, _f32, _i32, _vp, _i64,
                                                 _vp, _vp]),
        "mlp_deep_check_errors": (ctypes.c_int, [_vp]),
        "mlp_deep_profile": (ctypes.c_int, [_vp, _i32]),
        "mlp_deep_last_kernel_ms": (ctypes.c_int, [_vp, ctypes.POINTER(_f32)]),
        "mlp_deep_destroy": (None, [_vp]),
        "mlp_linear_workspace_bytes": (ctypes.c_size_t, [_i32, _i64, _i64, _i64]),
        "mlp_linear_init": (ctypes.c_int, [ctypes.POINTER(_vp), _i32, _i64, _i64, _i32, _i64, _vp,
                                           _vp, _vp, ctypes.c_size_t, _vp]),
        "mlp_linear_set_stream": (ctypes.c_int, [_vp, _vp]),
        "mlp_linear_forward": (ctypes.c_int, [_vp, _vp, _i64, _i64, _vp, _i64, _f32, _vp, _vp, _i64,
                                              _vp, _i64]),
        "mlp_linear_backward": (ctypes.c_int, [_vp, _vp, _i64, _vp, _i64, _vp, _i64, _i64, _f32, _vp,
                                               _vp, _i64, _vp, _vp]),
        "mlp_linear_destroy": (None, [_vp]),
        "mlp_dropout_forward": (ctypes.c_int, [_i32, _i64, _i64, _vp, _i64, _vp, _i64, _f32, _vp, _vp,
                                               _i64, _vp]),
        "mlp_dropout_backward": (ctypes.c_int, [_i32, _i64, _i64, _vp, _i64, _f32, _vp, _vp, _i64,
                                                _vp]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    return lib


def _check(fn, status):
    if status != MLP_OK:
        raise MLPError(fn, status)


def _dev(t, name, dtype=torch.float32, numel=None):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if numel is not None and t.numel() < numel:
        raise ValueError("%s has %d elements, needs %d" % (name, t.numel(), numel))
    return t.data_ptr()


def _stream(handle, device):
    """The stream of a handle; 0 is the device's default stream."""
    return torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device)


def _workspace(need, device, stream):
    """A workspace whose memory is in the order of the stream that clears and uses it: what is
    pending on another one may still write to a block of that one's pool."""
    with torch.cuda.stream(_stream(stream, device)):
        return torch.empty(need, dtype=torch.uint8, device=device)


def mlp_workspace_bytes(d_in: int, hidden: int, max_batch: int) -> int:
    return int(load().mlp_workspace_bytes(d_in, hidden, max_batch))


class Context:
    """A library context bound to caller-owned W1, W2 and workspace tensors."""

    def __init__(self, handle, W1, W2, workspace, max_batch, stream):
        self.handle = handle
        self.W1, self.W2, self.workspace = W1, W2, workspace
        self.stream = stream
        self.max_batch = max_batch
        self.hidden = W1.shape[1]
        self.strategy_workspace = None

    def __del__(self):
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.mlp_destroy(h)


def mlp_init(W1: torch.Tensor, W2: torch.Tensor, max_batch: int, workspace=None,
             stream=None) -> Context:
    """Create a context. W1 [32, h] and W2 [h] (or [h, 1]) are updated in place."""
    lib = load()
    if W1.dim() != 2:
        raise ValueError("W1 must be [d_in, hidden]")
    d_in, h = W1.shape
    _dev(W1, "W1")
    _dev(W2, "W2", numel=h)
    need = lib.mlp_workspace_bytes(d_in, h, max_batch)
    if need == 0:
        raise MLPError("mlp_workspace_bytes", -2)
    if stream is None:
        stream = torch.cuda.current_stream(W1.device).cuda_stream
    if workspace is None:
        workspace = _workspace(need, W1.device, stream)
    _dev(workspace, "workspace", dtype=torch.uint8, numel=need)
    handle = _vp()
    _check("mlp_init", lib.mlp_init(ctypes.byref(handle), d_in, h, 1, max_batch, W1.data_ptr(),
                                    W2.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                    stream))
    return Context(handle, W1, W2, workspace, max_batch, stream)


def mlp_set_stream(ctx: Context, stream) -> None:
    """Later calls go on `stream`, which the caller orders behind those before; it has to
    live as long as the context."""
    _check("mlp_set_stream", load().mlp_set_stream(ctx.handle, stream))
    ctx.stream = stream
    for w in (ctx.workspace, ctx.strategy_workspace):
        if w is not None:   # the allocator has to know of every stream that it was used on
            w.record_stream(_stream(stream, w.device))


def mlp_strategy_workspace_bytes(d_in: int, hidden: int, max_batch: int, strategy: int) -> int:
    return int(load().mlp_strategy_workspace_bytes(d_in, hidden, max_batch, strategy))


def mlp_set_strategy(ctx: Context, strategy, workspace=None) -> None:
    """Select the training strategy (a name of STRATEGIES or its code); allocates
    the strategy workspace as a torch tensor when none is given."""
    code = STRATEGIES[strategy] if isinstance(strategy, str) else int(strategy)
    need = mlp_strategy_workspace_bytes(D_IN, ctx.hidden, ctx.max_batch, code)
    if workspace is None and need > 0:
        workspace = _workspace(need, ctx.W1.device, ctx.stream)
    ptr = _dev(workspace, "workspace", dtype=torch.uint8, numel=need) if workspace is not None else None
    nbytes = workspace.numel() if workspace is not None else 0
    _check("mlp_set_strategy", load().mlp_set_strategy(ctx.handle, code, ptr, nbytes))
    ctx.strategy_workspace = workspace


def _rows(idx, B, name="idx"):
    if idx is None:
        return None
    return _dev(idx, name, dtype=torch.int32, numel=B)


def mlp_forward(ctx: Context, X, idx=None, B=None, out=None):
    n_rows = X.shape[0]
    B = (n_rows if idx is None else idx.numel()) if B is None else B
    _dev(X, "X", numel=n_rows * D_IN)
    if out is None:
        out = torch.empty(B, dtype=torch.float32, device=X.device)
    _check("mlp_forward", load().mlp_forward(ctx.handle, X.data_ptr(), n_rows, _rows(idx, B), B,
                                             _dev(out, "Ypred", numel=B)))
    return out


def mlp_backward(ctx: Context, X, Y, idx=None, B=None):
    n_rows = X.shape[0]
    B = (n_rows if idx is None else idx.numel()) if B is None else B
    _dev(X, "X", numel=n_rows * D_IN)
    _dev(Y, "Y", numel=n_rows)
    dW1 = torch.empty_like(ctx.W1)
    dW2 = torch.empty(ctx.hidden, dtype=torch.float32, device=X.device)
    loss = torch.empty(1, dtype=torch.float32, device=X.device)
    _check("mlp_backward", load().mlp_backward(ctx.handle, X.data_ptr(), n_rows, Y.data_ptr(),
                                               _rows(idx, B), B, dW1.data_ptr(), dW2.data_ptr(),
                                               loss.data_ptr()))
    return dW1, dW2, loss


def mlp_sgd_step(ctx: Context, X, Y, lr, idx=None, B=None, loss=None):
    n_rows = X.shape[0]
    B = (n_rows if idx is None else idx.numel()) if B is None else B
    _dev(X, "X", numel=n_rows * D_IN)
    _dev(Y, "Y", numel=n_rows)
    lp = _dev(loss, "loss", numel=1) if loss is not None else None
    _check("mlp_sgd_step", load().mlp_sgd_step(ctx.handle, X.data_ptr(), n_rows, Y.data_ptr(),
                                               _rows(idx, B), B, float(lr), lp))
    return loss


def mlp_train_epochs(ctx: Context, X, Y, batch, lr, epochs, perm=None, max_steps=-1,
                     epoch_loss=None, step_loss=None):
    n = X.shape[0]
    _dev(X, "X", numel=n * D_IN)
    _dev(Y, "Y", numel=n)
    pp = _dev(perm, "perm", dtype=torch.int32, numel=epochs * n) if perm is not None else None
    ep = _dev(epoch_loss, "epoch_loss", numel=epochs) if epoch_loss is not None else None
    steps = -(-n // batch) * epochs
    if max_steps >= 0:
        steps = min(steps, max_steps)
    sp = _dev(step_loss, "step_loss", numel=steps) if step_loss is not None else None
    _check("mlp_train_epochs", load().mlp_train_epochs(ctx.handle, X.data_ptr(), Y.data_ptr(), n,
                                                       batch, float(lr), epochs, pp, max_steps,
                                                       ep, sp))


def mlp_train_epochs_static(W1, W2, X, Y, batch, lr, epochs, perm=None, max_steps=-1,
                            epoch_loss=None, step_loss=None, status=None, stream=None):
    """mlp_train_epochs without a context: the library's own per-GPU scratch, no
    allocation in the call. W1 [32, h], W2 [h] are updated in place; status
    (nullable int32 [1]) receives the call's kernel-side error word."""
    if W1.dim() != 2:
        raise ValueError("W1 must be [d_in, hidden]")
    h = W1.shape[1]
    n = X.shape[0]
    _dev(W1, "W1")
    _dev(W2, "W2", numel=h)
    _dev(X, "X", numel=n * D_IN)
    _dev(Y, "Y", numel=n)
    pp = _dev(perm, "perm", dtype=torch.int32, numel=epochs * n) if perm is not None else None
    ep = _dev(epoch_loss, "epoch_loss", numel=epochs) if epoch_loss is not None else None
    steps = -(-n // batch) * epochs
    if max_steps >= 0:
        steps = min(steps, max_steps)
    sp = _dev(step_loss, "step_loss", numel=steps) if step_loss is not None else None
    stp = _dev(status, "status", dtype=torch.int32, numel=1) if status is not None else None
    if stream is None:
        stream = torch.cuda.current_stream(W1.device).cuda_stream
    _check("mlp_train_epochs_static",
           load().mlp_train_epochs_static(h, W1.data_ptr(), W2.data_ptr(), X.data_ptr(),
                                          Y.data_ptr(), n, batch, float(lr), epochs, pp,
                                          max_steps, ep, sp, stp, stream))


def mlp_check_errors(ctx: Context) -> None:
    _check("mlp_check_errors", load().mlp_check_errors(ctx.handle))


def mlp_profile(ctx: Context, enable: bool) -> None:
    _check("mlp_profile", load().mlp_profile(ctx.handle, 1 if enable else 0))


def mlp_last_kernel_ms(ctx: Context) -> float:
    ms = _f32(0.0)
    _check("mlp_last_kernel_ms", load().mlp_last_kernel_ms(ctx.handle, ctypes.byref(ms)))
    return float(ms.value)


def mlp_launch_info(ctx: Context, n, batch, epochs):
    wg = _i32(0)
    launches = _i64(0)
    _check("mlp_launch_info", load().mlp_launch_info(ctx.handle, n, batch, epochs,
                                                     ctypes.byref(wg), ctypes.byref(launches)))
    return int(wg.value), int(launches.value)


PHASE_NAMES = ("forward operands", "forward", "exchange A wait",
               "residual tile 0 (of two)", "residual + backward + P to LDS",
               "P barrier", "exchange B stores", "exchange B wait", "update + exchange C stores",
               "owners barrier", "exchange C gather", "step barrier")


def mlp_phase_cycles(ctx: Context):
    """Phase-cycle sums of the context's last fused-trainer call made with
    MLP_TRACE=1 (see include/mlp.h): an int64 array [workgroups, 2, 16], or None
    when no traced call wrote any."""
    import numpy as np
    words = _i64(0)
    _check("mlp_phase_cycles", load().mlp_phase_cycles(ctx.handle, None, 0, ctypes.byref(words)))
    if words.value <= 0:
        return None
    out = np.zeros(words.value, dtype=np.uint64)
    _check("mlp_phase_cycles", load().mlp_phase_cycles(ctx.handle, out.ctypes.data, words.value,
                                                       ctypes.byref(words)))
    return out.astype(np.int64).reshape(-1, 2, 16)


def mlp_status_string(status: int) -> str:
    return load().mlp_status_string(status).decode()


# --- deeper networks (L hidden layers) ------------------------------------------

def mlp_deep_param_count(d_in: int, hidden: int, layers: int) -> int:
    return int(load().mlp_deep_param_count(d_in, hidden, layers))


class DeepContext:
    """A deep-net context bound to caller-owned parameters and workspace."""

    def __init__(self, handle, params, workspace, hidden, layers, max_batch):
        self.handle = handle
        self.params, self.workspace = params, workspace
        self.hidden, self.layers, self.max_batch = hidden, layers, max_batch

    def __del__(self):
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.mlp_deep_destroy(h)


def mlp_deep_init(params: torch.Tensor, hidden: int, layers: int, max_batch: int,
                  workspace=None, stream=None) -> DeepContext:
    """params: flat fp32 [W_1 (32 x h) | W_2 .. W_L (h x h) | w_o (h)], updated in place."""
    lib = load()
    np_ = lib.mlp_deep_param_count(D_IN, hidden, layers)
    if np_ == 0:
        raise MLPError("mlp_deep_param_count", -2)
    _dev(params, "params", numel=np_)
    need = lib.mlp_deep_workspace_bytes(D_IN, hidden, layers, max_batch)
    if need == 0:
        raise MLPError("mlp_deep_workspace_bytes", -1)
    if stream is None:
        stream = torch.cuda.current_stream(params.device).cuda_stream
    if workspace is None:
        workspace = _workspace(need, params.device, stream)
    _dev(workspace, "workspace", dtype=torch.uint8)
    handle = _vp()
    # the library also takes a workspace without the part its panel path uses
    status = lib.mlp_deep_init(ctypes.byref(handle), D_IN, hidden, layers, 1, max_batch,
                               params.data_ptr(), workspace.data_ptr(), workspace.numel(), stream)
    if status == -3 and workspace.numel() < need:
        raise ValueError("workspace has %d elements, needs %d" % (workspace.numel(), need))
    _check("mlp_deep_init", status)
    return DeepContext(handle, params, workspace, hidden, layers, max_batch)


def mlp_deep_forward(ctx: DeepContext, X, idx=None, B=None, out=None):
    n_rows = X.shape[0]
    B = (n_rows if idx is None else idx.numel()) if B is None else B
    _dev(X, "X", numel=n_rows * D_IN)
    if out is None:
        out = torch.empty(B, dtype=torch.float32, device=X.device)
    _check("mlp_deep_forward", load().mlp_deep_forward(ctx.handle, X.data_ptr(), n_rows,
                                                       _rows(idx, B), B,
                                                       _dev(out, "Ypred", numel=B)))
    return out


def mlp_deep_backward(ctx: DeepContext, X, Y, idx=None, B=None):
    n_rows = X.shape[0]
    B = (n_rows if idx is None else idx.numel()) if B is None else B
    _dev(X, "X", numel=n_rows * D_IN)
    _dev(Y, "Y", numel=n_rows)
    dP = torch.empty_like(ctx.params)
    loss = torch.empty(1, dtype=torch.float32, device=X.device)
    _check("mlp_deep_backward", load().mlp_deep_backward(ctx.handle, X.data_ptr(), n_rows,
                                                         Y.data_ptr(), _rows(idx, B), B,
                                                         dP.data_ptr(), loss.data_ptr()))
    return dP, loss


def mlp_deep_sgd_step(ctx: DeepContext, X, Y, lr, idx=None, B=None, loss=None):
    n_rows = X.shape[0]
    B = (n_rows if idx is None else idx.numel()) if B is None else B
    _dev(X, "X", numel=n_rows * D_IN)
    _dev(Y, "Y", numel=n_rows)
    lp = _dev(loss, "loss", numel=1) if loss is not None else None
    _check("mlp_deep_sgd_step", load().mlp_deep_sgd_step(ctx.handle, X.data_ptr(), n_rows,
                                                         Y.data_ptr(), _rows(idx, B), B,
                                                         float(lr), lp))
    return loss


def mlp_deep_train_epochs(ctx: DeepContext, X, Y, batch, lr, epochs, perm=None, max_steps=-1,
                          epoch_loss=None, step_loss=None):
    n = X.shape[0]
    _dev(X, "X", numel=n * D_IN)
    _dev(Y, "Y", numel=n)
    pp = _dev(perm, "perm", dtype=torch.int32, numel=epochs * n) if perm is not None else None
    ep = _dev(epoch_loss, "epoch_loss", numel=epochs) if epoch_loss is not None else None
    steps = -(-n // batch) * epochs
    if max_steps >= 0:
        steps = min(steps, max_steps)
    sp = _dev(step_loss, "step_loss", numel=steps) if step_loss is not None else None
    _check("mlp_deep_train_epochs", load().mlp_deep_train_epochs(ctx.handle, X.data_ptr(),
                                                                 Y.data_ptr(), n, batch, float(lr),
                                                                 epochs, pp, max_steps, ep, sp))


def mlp_deep_check_errors(ctx: DeepContext) -> None:
    _check("mlp_deep_check_errors", load().mlp_deep_check_errors(ctx.handle))


def mlp_deep_profile(ctx: DeepContext, enable: bool) -> None:
    _check("mlp_deep_profile", load().mlp_deep_profile(ctx.handle, 1 if enable else 0))


def mlp_deep_last_kernel_ms(ctx: DeepContext) -> float:
    ms = _f32(0.0)
    _check("mlp_deep_last_kernel_ms", load().mlp_deep_last_kernel_ms(ctx.handle, ctypes.byref(ms)))
    return float(ms.value)


# --- layers: a dense layer and dropout -------------------------------------------

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
FIRST_ROWS = 1024   # room of a context whose caller names no max_rows
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


def _mat(t, name, dtype, device, rows, cols):
    """(pointer, row stride) of a [rows, cols] matrix whose rows are contiguous."""
    if t is None:
        return None, 0
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.device == device and t.shape == (rows, cols):
        sr, sc = t.stride()
        if (sc == 1 or cols <= 1) and (sr >= cols or rows <= 1):
            return t.data_ptr(), (sr if rows > 1 else cols)
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    if t.device != device:
        raise ValueError("%s is on %s, not on %s" % (name, t.device, device))
    if t.shape != (rows, cols):
        raise ValueError("%s must be [%d, %d], is %s" % (name, rows, cols, list(t.shape)))
    if cols > 1 and t.stride(1) != 1:
        raise ValueError("the elements of a row of %s must be adjacent" % name)
    raise ValueError("the rows of %s overlap" % name)


def _vec(t, name, dtype, device, n):
    if t is None:
        return None
    p = _dev(t, name, dtype=dtype)
    if t.device != device:
        raise ValueError("%s is on %s, not on %s" % (name, t.device, device))
    if t.numel() != n:
        raise ValueError("%s has %d elements, needs %d" % (name, t.numel(), n))
    return p


def _rng(rng, device):
    """The generator's state: int64 [2] (seed, offset) in device memory."""
    return None if rng is None else _vec(rng, "rng", torch.int64, device, 2)


# The handle of the stream that is current on a device. (A call of a small layer takes
# about 7 us of the host, half of it the launch; torch.cuda.current_stream, which makes an
# object of the handle, would add 1.8.)
_current_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


class LinearContext:
    """A dense layer's context bound to caller-owned W, bias and workspace."""

    def __init__(self, handle, W, bias, workspace, activation, max_rows, stream, bound, grows=False):
        self.handle = handle
        self.W, self.bias, self.workspace = W, bias, workspace
        self.d_in, self.d_out = W.shape
        self.dtype, self.device = W.dtype, W.device
        self.activation, self.max_rows = activation, max_rows
        self.stream = stream    # None: each call goes on the current stream
        self.bound = bound      # the stream the library's context is on
        self.last = bound       # the stream of the last call that was not captured
        self.grows = grows      # whether calls of more than max_rows rows make room
        self.before = []        # the smaller workspaces before this one

    def __del__(self):
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.mlp_linear_destroy(h)


def mlp_linear_workspace_bytes(dtype: torch.dtype, d_in: int, d_out: int, max_rows: int) -> int:
    return int(load().mlp_linear_workspace_bytes(DTYPES[dtype], d_in, d_out, max_rows))


def _linear_context(W, bias, activation, max_rows, workspace, stream):
    """(handle, workspace) of a context of the library's on `stream`."""
    lib = load()
    d_in, d_out = W.shape
    wp = _dev(W, "W", dtype=W.dtype)
    bp = _vec(bias, "bias", W.dtype, W.device, d_out)
    need = mlp_linear_workspace_bytes(W.dtype, d_in, d_out, max_rows)
    if need == 0:
        raise MLPError("mlp_linear_workspace_bytes", -2)
    with torch.cuda.device(W.device):
        if workspace is None:
            workspace = _workspace(need, W.device, stream)
        if workspace.device != W.device:
            raise ValueError("workspace is on %s, not on %s" % (workspace.device, W.device))
        _dev(workspace, "workspace", dtype=torch.uint8, numel=need)
        handle = _vp()
        _check("mlp_linear_init",
               lib.mlp_linear_init(ctypes.byref(handle), DTYPES[W.dtype], d_in, d_out,
                                   ACTIVATIONS[activation], max_rows, wp, bp, workspace.data_ptr(),
                                   workspace.numel(), stream))
    return handle, workspace


def mlp_linear_init(W: torch.Tensor, bias=None, activation="none", max_rows=None, workspace=None,
                    stream=None) -> LinearContext:
    """A dense layer y = residual + dropout(a(X W + bias)). W [d_in, d_out] (float32,
    bfloat16 or float16), bias [d_out] or None; activation a name of ACTIVATIONS.
    max_rows: the most rows of a call, which the workspace's size goes by; without it there is
    room for 1,024 rows, and a call of more, unless it is captured, makes room for them (with a
    workspace of the caller's it is the most there may be, 2^20). Calls go on `stream`, or on the current stream at each
    call where none is given; a caller's workspace is taken to be free there (several layers
    may share one, if their calls do not overlap: over streams the caller orders those). A
    HIP graph that holds calls replays them on the context's workspace: keep the context as
    long as the graph."""
    if W.dim() != 2:
        raise ValueError("W must be [d_in, d_out]")
    if W.dtype not in DTYPES:
        raise TypeError("W must be one of %s" % (tuple(DTYPES),))
    _dev(W, "W", dtype=W.dtype)
    grows = max_rows is None and workspace is None
    if max_rows is None:
        max_rows = FIRST_ROWS if grows else MAX_BATCH
    bound = torch.cuda.current_stream(W.device).cuda_stream if stream is None else stream
    handle, workspace = _linear_context(W, bias, activation, max_rows, workspace, bound)
    return LinearContext(handle, W, bias, workspace, activation, max_rows, stream, bound, grows)


def _grow(ctx, rows):
    """Room for `rows` rows, as a power of two (what the library refuses stays refused). Captured
    calls replay on the workspaces before, which are kept."""
    with torch.cuda.device(ctx.device), torch.cuda.stream(_stream(ctx.bound, ctx.device)):
        if rows > MAX_BATCH or torch.cuda.is_current_stream_capturing():
            return
    most = 1 << (rows - 1).bit_length()
    handle, workspace = _linear_context(ctx.W, ctx.bias, ctx.activation, most, None, ctx.bound)
    load().mlp_linear_destroy(ctx.handle)
    ctx.before.append(ctx.workspace)
    ctx.handle, ctx.workspace, ctx.max_rows = handle, workspace, most


def mlp_linear_set_stream(ctx: LinearContext, stream) -> None:
    """Later calls go on `stream` (None: on the current stream at each call), behind those
    before. The stream has to live as long as the context."""
    if stream is not None:
        _move(ctx, stream)
    ctx.stream = stream


def _move(ctx, now):
    """Put the context on the stream `now`, behind the calls it made on another one before
    (a stream that captures cannot wait for those: there the capture's own start has to be
    behind them, and the next call that is not captured still waits). When the context is
    dropped, maybe with calls under way, its workspace goes back to the allocator, which has
    to know of every stream that it was used on."""
    at = _stream(now, ctx.device)
    with torch.cuda.device(ctx.device), torch.cuda.stream(at):
        captured = torch.cuda.is_current_stream_capturing()
    if now != ctx.last and not captured:
        at.wait_stream(_stream(ctx.last, ctx.device))
        ctx.last = now
    if now != ctx.bound:
        ctx.workspace.record_stream(at)
        _check("mlp_linear_set_stream", load().mlp_linear_set_stream(ctx.handle, now))
        ctx.bound = now


def _bind_stream(ctx):
    """Put the context on the current stream where it has none of its own."""
    if ctx.stream is None:
        now = _current_stream(ctx.device.index)
        if now != ctx.bound or now != ctx.last:
            _move(ctx, now)


def _new(ctx, *shape):
    """An output of the context's type, its memory taken on the stream that writes it."""
    if ctx.stream is None:
        return torch.empty(shape, dtype=ctx.dtype, device=ctx.device)
    with torch.cuda.stream(_stream(ctx.stream, ctx.device)):
        return torch.empty(shape, dtype=ctx.dtype, device=ctx.device)


def mlp_linear_forward(ctx: LinearContext, X, residual=None, p=0.0, rng=None, out=None, z=None,
                       save_z=False):
    """Y = residual + dropout(a(X W + bias)); with save_z (or a tensor z) also z = X W +
    bias, which the backward call takes: then (Y, z) is returned."""
    if X.dim() != 2:
        raise ValueError("X must be [rows, d_in]")
    rows, n, dev, dt = X.shape[0], ctx.d_out, ctx.device, ctx.dtype
    xp, ldx = _mat(X, "X", dt, dev, rows, ctx.d_in)
    rp, ldr = _mat(residual, "residual", dt, dev, rows, n)
    gp = _rng(rng, dev)
    if out is None:
        out = _new(ctx, rows, n)
    if z is None and save_z:
        z = _new(ctx, rows, n)
    yp, ldy = _mat(out, "out", dt, dev, rows, n)
    zp, ldz = _mat(z, "z", dt, dev, rows, n)
    _bind_stream(ctx)
    if rows > ctx.max_rows and ctx.grows:
        _grow(ctx, rows)
    _check("mlp_linear_forward", load().mlp_linear_forward(ctx.handle, xp, ldx, rows, rp, ldr, float(p), gp, yp,
                                                           ldy, zp, ldz))
    return out if z is None else (out, z)


def mlp_linear_backward(ctx: LinearContext, X, dY, z=None, p=0.0, rng=None, need_dx=True, need_dw=True,
                        need_db=True, dX=None, dW=None, db=None):
    """(dX, dW, db) of a forward call with the same X, p and rng; None for what is not
    needed (db: for a layer without bias). X may be None where dW is not needed. A dW of the
    caller's is [d_in, d_out] or flat."""
    if dY.dim() != 2:
        raise ValueError("dY must be [rows, d_out]")
    rows, n, dev, dt = dY.shape[0], ctx.d_out, ctx.device, ctx.dtype
    xp, ldx = _mat(X, "X", dt, dev, rows, ctx.d_in)
    gyp, lddy = _mat(dY, "dY", dt, dev, rows, n)
    zp, ldz = _mat(z, "z", dt, dev, rows, n)
    gp = _rng(rng, dev)
    if dW is not None and dW.dim() != 1 and dW.shape != (ctx.d_in, n):   # (flat: a slice of a bucket)
        raise ValueError("dW must be [%d, %d], is %s" % (ctx.d_in, n, list(dW.shape)))
    if dX is None and need_dx:
        dX = _new(ctx, rows, ctx.d_in)
    if dW is None and need_dw:
        dW = _new(ctx, ctx.d_in, n)
    if db is None and need_db and ctx.bias is not None:
        db = _new(ctx, n)
    dxp, lddx = _mat(dX, "dX", dt, dev, rows, ctx.d_in)
    dwp = _vec(dW, "dW", dt, dev, ctx.d_in * n)
    dbp = _vec(db, "db", dt, dev, n)
    _bind_stream(ctx)
    if rows > ctx.max_rows and ctx.grows:
        _grow(ctx, rows)
    _check("mlp_linear_backward",
           load().mlp_linear_backward(ctx.handle, xp, ldx, zp, ldz, gyp, lddy, rows, float(p), gp,
                                      dxp, lddx, dwp, dbp))
    return dX, dW, db


def _dropout_call(fn, X, p, rng, residual, out, name):
    if X.dim() != 2:
        raise ValueError("%s must be [rows, cols]" % name)
    dev, dt = X.device, X.dtype
    if dt not in DTYPES:
        raise TypeError("%s must be one of %s" % (name, tuple(DTYPES)))
    if not X.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) tensor" % name)
    p = float(p)
    if p == 0.0 and out is None and residual is None:
        return X
    rows, cols = X.shape
    xp, ldx = _mat(X, name, dt, dev, rows, cols)
    rp, ldr = _mat(residual, "residual", dt, dev, rows, cols)
    gp = _rng(rng, dev)
    if out is None:
        out = torch.empty((rows, cols), dtype=dt, device=dev)
        yp, ldy = out.data_ptr(), cols
    else:
        yp, ldy = _mat(out, "out", dt, dev, rows, cols)
    args = (xp, ldx, p, gp, yp, ldy)
    if fn == "mlp_dropout_forward":
        args = (xp, ldx, rp, ldr, p, gp, yp, ldy)
    f, s = getattr(load(), fn), _current_stream(dev.index)
    if dev.index == torch.cuda.current_device():
        st = f(DTYPES[dt], rows, cols, *args, s)
    else:
        with torch.cuda.device(dev):
            st = f(DTYPES[dt], rows, cols, *args, s)
    _check(fn, st)
    return out


def mlp_dropout_forward(X, p, rng, residual=None, out=None):
    """residual + dropout(X) on the current stream of X's device; rng int64 [2] (seed,
    offset) in device memory. out may be X or residual. With p = 0, no residual and no out
    the result is X itself."""
    return _dropout_call("mlp_dropout_forward", X, p, rng, residual, out, "X")


def mlp_dropout_backward(dY, p, rng, out=None):
    """The gradient of mlp_dropout_forward with the same p and rng; out may be dY. With p =
    0 and no out the result is dY itself."""
    return _dropout_call("mlp_dropout_backward", dY, p, rng, None, out, "dY")
