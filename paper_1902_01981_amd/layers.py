"""ctypes binding with the names of include/codedreduce_layers.h.

Every function marshals its arguments and calls the C-ABI entry point of the same name; all arithmetic runs in the HIP library.
Activations are torch tensors of shape (points, channels), (points, positions, channels) or with more dimensions of positions that can be
viewed as one; channels are contiguous, the other strides are the tensor's own.  All tensors live on the current device.  Launches go to
torch's current stream unless another one is given; where a call needs a workspace and is given none, it takes one from torch's allocator.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

from .api import CR_BF16, CR_F32, CR_OK, CodedReduceError

_HERE = os.path.dirname(os.path.abspath(__file__))
LAYERS_LIB_PATH = os.path.join(_HERE, "libcodedreduce_layers.so")

CR_ACT_NONE, CR_ACT_RELU, CR_ACT_SILU = 0, 1, 2

LAYERS_EXPORTS = ["cr_layers_last_error", "cr_group_norm_workspace_bytes", "cr_group_norm_forward", "cr_group_norm_backward",
                  "cr_dropout_workspace_bytes", "cr_dropout_forward", "cr_dropout_backward", "cr_softmax_loss_workspace_bytes", "cr_softmax_loss"]


class cr_layer_shape_t(ctypes.Structure):
    _fields_ = [("points", ctypes.c_int64), ("positions", ctypes.c_int64), ("channels", ctypes.c_int64), ("dtype", ctypes.c_int32)]


class cr_layer_view_t(ctypes.Structure):
    _fields_ = [("dev", ctypes.c_void_p), ("point_stride", ctypes.c_int64), ("position_stride", ctypes.c_int64)]


class cr_dropout_t(ctypes.Structure):
    _fields_ = [("rate", ctypes.c_double), ("seed", ctypes.c_uint64), ("draw", ctypes.c_uint64), ("draw_dev", ctypes.c_void_p),
                ("first_point", ctypes.c_int64), ("point_dev", ctypes.c_void_p)]


_lib = None


def load_layers_library():
    """Loads the built shared library; raises if it is missing (there is no other implementation to fall back to)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LAYERS_LIB_PATH):
            raise ImportError(f"{LAYERS_LIB_PATH} is not built: run `python paper_1902_01981_amd/build.py`")
        lib = ctypes.CDLL(LAYERS_LIB_PATH)
        vp, i64, c_int, size_t = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
        shape, view, drop, size_p = ctypes.POINTER(cr_layer_shape_t), ctypes.POINTER(cr_layer_view_t), ctypes.POINTER(cr_dropout_t), ctypes.POINTER(size_t)
        lib.cr_layers_last_error.restype = ctypes.c_char_p
        lib.cr_group_norm_workspace_bytes.argtypes = [shape, c_int, vp, c_int, size_p, size_p]
        lib.cr_group_norm_forward.argtypes = [shape, view, vp, vp, c_int, ctypes.c_float, c_int, view, vp, vp, vp, size_t, vp]
        lib.cr_group_norm_backward.argtypes = [shape, view, view, vp, vp, vp, vp, c_int, c_int, vp, c_int, view, vp, vp, vp, size_t, vp]
        lib.cr_dropout_workspace_bytes.argtypes = [shape, vp, c_int, size_p]
        lib.cr_dropout_forward.argtypes = [shape, view, vp, view, drop, view, vp]
        lib.cr_dropout_backward.argtypes = [shape, view, drop, view, vp, c_int, vp, vp, size_t, vp]
        lib.cr_softmax_loss_workspace_bytes.argtypes = [i64, i64, c_int, size_p]
        lib.cr_softmax_loss.argtypes = [i64, i64, c_int, vp, i64, vp, vp, vp, vp, vp, i64, vp, size_t, vp]
        _lib = lib
    return _lib


def cr_layers_last_error() -> str:
    return load_layers_library().cr_layers_last_error().decode()


def _check(status: int) -> None:
    if status != CR_OK:
        raise CodedReduceError(status, cr_layers_last_error())


_DTYPES = {torch.float32: CR_F32, torch.bfloat16: CR_BF16}


# A call takes the host as long as its launch does (4 us) and what is marshalled here: these two without the objects that torch.cuda makes of them (0.1 us
# in place of 3 for a stream).
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _on_device(t, name: str) -> None:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    device = t.get_device()                              # -1: not on a GPU
    if device < 0 or device != _current_device():
        raise ValueError(f"{name} must live on the current GPU")


def _shape_of(t, name: str) -> cr_layer_shape_t:
    _on_device(t, name)
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name} has dtype {t.dtype}, expected torch.float32 or torch.bfloat16")
    size = t.shape
    if len(size) < 2:
        raise ValueError(f"{name} must have the shape (points, positions ..., channels)")
    positions = 1
    for n in size[1:-1]:
        positions *= n
    return cr_layer_shape_t(size[0], positions, size[-1], _DTYPES[t.dtype])


def _view(t, like, name: str):
    """The view of an activation that has the shape and type of `like`."""
    if t is not like:
        _on_device(t, name)
        if t.shape != like.shape or t.dtype != like.dtype:
            raise ValueError(f"{name} has shape {tuple(t.shape)} and dtype {t.dtype}, expected {tuple(like.shape)} and {like.dtype}")
    strides = t.stride()
    if strides[-1] != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name} must have contiguous channels")
    if len(strides) == 3:
        position = strides[1]
    elif len(strides) == 2:
        position = 0
    else:                                                # several dimensions of positions: one stride must serve them all
        position, size = None, 1
        for n, stride in zip(reversed(t.shape[1:-1]), reversed(strides[1:-1])):
            if n == 1:
                continue
            if position is None:
                position = stride
            elif stride != position * size:
                raise ValueError(f"{name}: its positions cannot be viewed as one dimension")
            size *= n
        position = position or 0
    return cr_layer_view_t(t.data_ptr(), strides[0], position)


def _vector(t, count: int, name: str, dtype=torch.float32, optional: bool = True) -> int:
    """Address of a contiguous device tensor of `count` elements."""
    if t is None:
        if optional:
            return 0
        raise ValueError(f"{name} is required")
    _on_device(t, name)
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.numel() != count or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous and have {count} elements")
    return t.data_ptr()


def _bounds(bounds):
    """(address, runs, what keeps the address alive) of the runs' bounds."""
    if bounds is None:
        return 0, 1, None
    given = np.asarray(bounds)
    if given.ndim != 1 or given.size < 2:
        raise ValueError("bounds must be runs + 1 numbers")
    if given.dtype.kind not in "iu" and not ((np.abs(given) < 2.0 ** 62).all() and (np.mod(given, 1) == 0).all()):
        raise ValueError("bounds must be whole numbers")
    b = np.ascontiguousarray(given, dtype=np.int64)
    return b.ctypes.data, b.size - 1, b


def _stream(stream) -> int:
    """The stream of a call: the one given, else torch's current one."""
    if stream is not None:
        return stream
    return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(_current_device())


def _workspace(workspace, nbytes: int, stream):
    """(address, bytes, what keeps it alive) of a workspace of at least nbytes."""
    if nbytes == 0:
        return 0, 0, None
    if workspace is None:
        if stream is not None and stream != _stream(None):
            raise ValueError("a call on another stream than torch's current one brings its own workspace")
        workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    else:
        _on_device(workspace, "workspace")
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


# ---- group norm with an activation ---------------------------------------------------------------------------------------
def cr_group_norm_workspace_bytes(x, groups: int, bounds=None):
    """(bytes of the forward pass, bytes of the backward pass) for activations like x."""
    f, b = ctypes.c_size_t(), ctypes.c_size_t()
    at, runs, _keep = _bounds(bounds)
    _check(load_layers_library().cr_group_norm_workspace_bytes(_shape_of(x, "x"), groups, at, runs, ctypes.byref(f), ctypes.byref(b)))
    return f.value, b.value


def cr_group_norm_forward(x, gamma, beta, groups: int, y, mean=None, rstd=None, eps: float = 1e-5, activation: int = CR_ACT_NONE,
                          workspace=None, stream=None) -> None:
    lib = load_layers_library()
    shape = _shape_of(x, "x")
    need, unused = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib.cr_group_norm_workspace_bytes(shape, groups, 0, 1, ctypes.byref(need), ctypes.byref(unused)))
    ws, nbytes, _keep = _workspace(workspace, need.value, stream)
    stats = shape.points * groups
    _check(lib.cr_group_norm_forward(shape, _view(x, x, "x"), _vector(gamma, shape.channels, "gamma"), _vector(beta, shape.channels, "beta"), groups,
                                     eps, activation, _view(y, x, "y"), _vector(mean, stats, "mean"), _vector(rstd, stats, "rstd"), ws, nbytes,
                                     _stream(stream)))


def cr_group_norm_backward(dy, x, mean, rstd, gamma, beta, groups: int, dx=None, dgamma=None, dbeta=None, activation: int = CR_ACT_NONE,
                           bounds=None, workspace=None, stream=None) -> None:
    lib = load_layers_library()
    shape = _shape_of(x, "x")
    at, runs, _keep = _bounds(bounds)
    unused, need = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib.cr_group_norm_workspace_bytes(shape, groups, at, runs, ctypes.byref(unused), ctypes.byref(need)))
    ws, nbytes, _keep_ws = _workspace(workspace, need.value, stream)
    stats, C = shape.points * groups, shape.channels
    _check(lib.cr_group_norm_backward(shape, _view(dy, x, "dy"), _view(x, x, "x"), _vector(mean, stats, "mean", optional=False),
                                      _vector(rstd, stats, "rstd", optional=False), _vector(gamma, C, "gamma"), _vector(beta, C, "beta"), groups,
                                      activation, at, runs, None if dx is None else _view(dx, x, "dx"), _vector(dgamma, runs * C, "dgamma"),
                                      _vector(dbeta, runs * C, "dbeta"), ws, nbytes, _stream(stream)))


# ---- bias, dropout, residual ---------------------------------------------------------------------------------------------
def _dropout(shape, rate, seed, draw, first_point, point_index, draw_dev) -> cr_dropout_t:
    return cr_dropout_t(rate, seed % (1 << 64), draw % (1 << 64), _vector(draw_dev, 1, "draw_dev", torch.int64), first_point,
                        _vector(point_index, shape.points, "point_index", torch.int64))


def cr_dropout_workspace_bytes(x, bounds=None) -> int:
    b = ctypes.c_size_t()
    at, runs, _keep = _bounds(bounds)
    _check(load_layers_library().cr_dropout_workspace_bytes(_shape_of(x, "x"), at, runs, ctypes.byref(b)))
    return b.value


def cr_dropout_forward(x, y, rate: float, seed: int, draw: int = 0, bias=None, residual=None, first_point: int = 0, point_index=None,
                       draw_dev=None, stream=None) -> None:
    """point_index: int64 indices of the points, in place of first_point, first_point + 1, ...; draw_dev: one int64 that is added to draw."""
    shape = _shape_of(x, "x")
    _check(load_layers_library().cr_dropout_forward(shape, _view(x, x, "x"), _vector(bias, shape.channels, "bias"),
                                                    None if residual is None else _view(residual, x, "residual"),
                                                    _dropout(shape, rate, seed, draw, first_point, point_index, draw_dev), _view(y, x, "y"),
                                                    _stream(stream)))


def cr_dropout_backward(dy, dx, rate: float, seed: int, draw: int = 0, dbias=None, bounds=None, first_point: int = 0, point_index=None,
                        draw_dev=None, workspace=None, stream=None) -> None:
    lib = load_layers_library()
    shape = _shape_of(dy, "dy")
    at, runs, _keep = _bounds(bounds)
    need = ctypes.c_size_t()
    if dbias is not None:
        _check(lib.cr_dropout_workspace_bytes(shape, at, runs, ctypes.byref(need)))
    ws, nbytes, _keep_ws = _workspace(workspace, need.value, stream)
    _check(lib.cr_dropout_backward(shape, _view(dy, dy, "dy"), _dropout(shape, rate, seed, draw, first_point, point_index, draw_dev),
                                   None if dx is None else _view(dx, dy, "dx"), at, runs, _vector(dbias, runs * shape.channels, "dbias"), ws, nbytes,
                                   _stream(stream)))


# ---- softmax loss --------------------------------------------------------------------------------------------------------
def cr_softmax_loss_workspace_bytes(rows: int, classes: int, dtype: int) -> int:
    b = ctypes.c_size_t()
    _check(load_layers_library().cr_softmax_loss_workspace_bytes(rows, classes, dtype, ctypes.byref(b)))
    return b.value


def cr_softmax_loss(logits, targets, loss, lse=None, dlogits=None, weights=None, workspace=None, stream=None) -> None:
    """logits (rows, classes); dlogits may be logits itself."""
    shape = _shape_of(logits, "logits")
    if logits.dim() != 2:
        raise ValueError("logits must have the shape (rows, classes)")
    rows, classes = shape.points, shape.channels
    x = _view(logits, logits, "logits")
    dx = cr_layer_view_t(0, 0, 0) if dlogits is None else _view(dlogits, logits, "dlogits")
    ws, nbytes, _keep = _workspace(workspace, cr_softmax_loss_workspace_bytes(rows, classes, shape.dtype), stream)
    _check(load_layers_library().cr_softmax_loss(rows, classes, shape.dtype, x.dev, x.point_stride, _vector(targets, rows, "targets", torch.int64, False),
                                                 _vector(weights, rows, "weights"), _vector(loss, rows, "loss", optional=False),
                                                 _vector(lse, rows, "lse"), dx.dev, dx.point_stride, ws, nbytes, _stream(stream)))
