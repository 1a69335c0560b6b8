"""Python binding of the dense layers (include/embx_dense.h): argument marshalling only.

    y = linear(x, weight, bias, residual, activation="relu")
    dx, dw, db = linear_backward(dy, x, weight, z, activation="relu")
    h = gated_ffn(x, w_gate, w_up, b_gate, b_up, activation="silu")
    dx, dw_gate, dw_up, db_gate, db_up = gated_ffn_backward(dh, x, w_gate, w_up, g, u)

Matrices are 2-D device tensors whose rows are contiguous (any row stride of at least a row),
vectors contiguous 1-D ones, all of one dtype: float32, float16 or bfloat16.  Results are
allocated (torch's allocator) unless ``out`` is given; calls run on ``stream`` (a
torch.cuda.Stream or a raw handle), the current stream by default.
"""
from __future__ import annotations

import ctypes

import torch

from . import OK, EmbxError, _current_stream_ptr, _i32, _i64, _lib, _sz, _vp

ACTIVATIONS = {"none": 0, "relu": 1, "sigmoid": 2, "silu": 3, "gelu": 4}
_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def _matrices(*names):
    return [f for name in names for f in ((name, _vp), ("ld_" + name, _i64))]


_SHAPE = [("m", _i64), ("n", _i64), ("k", _i64), ("dtype", _i32), ("activation", _i32)]


class _Linear(ctypes.Structure):
    _fields_ = _SHAPE + _matrices("x", "weight") + [("bias", _vp)] + _matrices("residual", "y", "z")


class _LinearGrad(ctypes.Structure):
    _fields_ = _SHAPE + _matrices("dy", "x", "weight", "z", "dx", "dweight") + [("dbias", _vp)]


class _Gated(ctypes.Structure):
    _fields_ = _SHAPE + _matrices("x", "w_gate", "w_up") + [("b_gate", _vp), ("b_up", _vp)] + _matrices("h", "g", "u")


class _GatedGrad(ctypes.Structure):
    _fields_ = _SHAPE + _matrices("dh", "x", "w_gate", "w_up", "g", "u", "dx", "dw_gate", "dw_up") \
        + [("db_gate", _vp), ("db_up", _vp)]


def _entry(name, struct):
    size = getattr(_lib, name + "_workspace")
    size.restype, size.argtypes = _i32, [ctypes.POINTER(struct), ctypes.POINTER(_sz)]
    fn = getattr(_lib, name)
    fn.restype, fn.argtypes = _i32, [ctypes.POINTER(struct), _vp, _sz, _vp]

    def call(a, device, stream):
        nbytes = _sz(0)
        code = size(a, nbytes)
        if code != OK:
            raise EmbxError(code, name)
        nbytes = nbytes.value
        ws = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
        code = fn(a, ws.data_ptr() if nbytes else None, nbytes, stream)
        if code != OK:
            raise EmbxError(code, name)

    return call


_linear, _linear_backward = _entry("emb_linear", _Linear), _entry("emb_linear_backward", _LinearGrad)
_gated, _gated_backward = _entry("emb_gated", _Gated), _entry("emb_gated_backward", _GatedGrad)


def _activation(name) -> int:
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}, got {name!r}") from None


def _first(x, name):
    """(rows, columns, dtype code, device) of the matrix that the others are measured against."""
    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dim() == 2):
        raise ValueError(f"{name} must be a 2-D device tensor")
    dtype = _DTYPES.get(x.dtype)
    if dtype is None:
        raise ValueError(f"{name} must be float32, float16 or bfloat16, got {x.dtype}")
    if x.get_device() != torch.cuda.current_device():
        raise ValueError(f"{name} is on {x.device}, the current device is cuda:{torch.cuda.current_device()}")
    return x.shape[0], x.shape[1], dtype, x.device


def _matrix(t, name, rows, cols, like):
    """(pointer, row stride) of a matrix [rows, cols] of like's dtype on its device."""
    if not (isinstance(t, torch.Tensor) and t.dtype == like.dtype and t.device == like.device and t.dim() == 2):
        raise ValueError(f"{name} must be a 2-D {like.dtype} tensor on {like.device}")
    if t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{name} must be [{rows}, {cols}], got {list(t.shape)}")
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{name} must have contiguous rows, got strides {t.stride()}")
    if rows <= 1:
        ld = cols if ld < cols else ld
    elif ld < cols:
        raise ValueError(f"{name}: rows must not overlap, got strides {t.stride()}")
    return t.data_ptr(), ld


def _rows(t, name):
    if not (isinstance(t, torch.Tensor) and t.dim() == 2):
        raise ValueError(f"{name} must be a 2-D device tensor")
    return t.shape[0]


def _vector(t, name, n, like):
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.dtype == like.dtype and t.device == like.device and t.dim() == 1
            and t.shape[0] == n and (n == 1 or t.stride(0) == 1)):
        raise ValueError(f"{name} must be a contiguous [{n}] {like.dtype} tensor on {like.device}")
    return t.data_ptr()


def _on(stream, fn, *args):
    """fn(raw stream handle, *args) with torch's allocations on that stream."""
    if stream is None:
        return fn(_current_stream_ptr(), *args)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    with torch.cuda.stream(stream):
        return fn(stream.cuda_stream, *args)


def linear(x, weight, bias=None, residual=None, *, activation="none", out=None, save=False, stream=None):
    """act(x weight^T + bias) + residual (emb_linear).  x [m, k], weight [n, k], bias [n],
    residual [m, n]; ``save``: also returns the sums before the activation, as
    linear_backward takes them.  ``out`` may be the residual."""
    return _on(stream, _run_linear, x, weight, bias, residual, activation, out, save)


def _run_linear(stream, x, weight, bias, residual, activation, out, save):
    act = _activation(activation)
    m, k, dtype, device = _first(x, "x")
    n = _rows(weight, "weight")
    y = torch.empty((m, n), dtype=x.dtype, device=device) if out is None else out
    z = torch.empty((m, n), dtype=x.dtype, device=device) if save else None
    a = _Linear(m, n, k, dtype, act, *_matrix(x, "x", m, k, x), *_matrix(weight, "weight", n, k, x),
                _vector(bias, "bias", n, x), *(_matrix(residual, "residual", m, n, x) if residual is not None else (None, 0)),
                *((y.data_ptr(), n) if out is None else _matrix(y, "out", m, n, x)),
                *((z.data_ptr(), n) if save else (None, 0)))
    _linear(a, device, stream)
    return (y, z) if save else y


def linear_backward(dy, x, weight, z=None, *, activation="none", bias=True, stream=None, need_dx=True, need_dw=True):
    """Gradients (dx, dweight, dbias) of linear at the gradient dy of its result (None where
    not wanted); z as linear(..., save=True) returned it (not needed with activation
    "none").  The residual's gradient is dy."""
    return _on(stream, _run_linear_backward, dy, x, weight, z, activation, bias, need_dx, need_dw)


def _run_linear_backward(stream, dy, x, weight, z, activation, bias, need_dx, need_dw):
    act = _activation(activation)
    m, k, dtype, device = _first(x, "x")
    n = _rows(weight, "weight")
    if act and z is None:
        raise ValueError(f"activation {activation!r} needs z, the sums that linear(..., save=True) returns")
    dx = torch.empty((m, k), dtype=x.dtype, device=device) if need_dx else None
    dw = torch.empty((n, k), dtype=x.dtype, device=device) if need_dw else None
    db = torch.empty(n, dtype=x.dtype, device=device) if bias else None
    a = _LinearGrad(m, n, k, dtype, act, *_matrix(dy, "dy", m, n, x), *_matrix(x, "x", m, k, x),
                    *_matrix(weight, "weight", n, k, x), *(_matrix(z, "z", m, n, x) if act else (None, 0)),
                    *((dx.data_ptr(), k) if need_dx else (None, 0)), *((dw.data_ptr(), k) if need_dw else (None, 0)),
                    db.data_ptr() if bias else None)
    _linear_backward(a, device, stream)
    return dx, dw, db


def gated_ffn(x, w_gate, w_up, b_gate=None, b_up=None, *, activation="silu", out=None, save=False, stream=None):
    """act(x w_gate^T + b_gate) * (x w_up^T + b_up) (emb_gated).  x [m, k], weights [n, k],
    biases [n]; ``save``: returns (h, g, u) with both projections, as gated_ffn_backward takes them."""
    return _on(stream, _run_gated, x, w_gate, w_up, b_gate, b_up, activation, out, save)


def _run_gated(stream, x, w_gate, w_up, b_gate, b_up, activation, out, save):
    act = _activation(activation)
    m, k, dtype, device = _first(x, "x")
    n = _rows(w_gate, "w_gate")
    h = torch.empty((m, n), dtype=x.dtype, device=device) if out is None else out
    g, u = (torch.empty((2, m, n), dtype=x.dtype, device=device) if save else (None, None))
    a = _Gated(m, n, k, dtype, act, *_matrix(x, "x", m, k, x), *_matrix(w_gate, "w_gate", n, k, x),
               *_matrix(w_up, "w_up", n, k, x), _vector(b_gate, "b_gate", n, x), _vector(b_up, "b_up", n, x),
               *((h.data_ptr(), n) if out is None else _matrix(h, "out", m, n, x)),
               *((g.data_ptr(), n, u.data_ptr(), n) if save else (None, 0, None, 0)))
    _gated(a, device, stream)
    return (h, g, u) if save else h


def gated_ffn_backward(dh, x, w_gate, w_up, g, u, *, activation="silu", bias=False, stream=None, need_dx=True,
                       need_dw=True):
    """Gradients (dx, dw_gate, dw_up, db_gate, db_up) of gated_ffn at the gradient dh of its
    result (None where not wanted); g and u as gated_ffn(..., save=True) returned them."""
    return _on(stream, _run_gated_backward, dh, x, w_gate, w_up, g, u, activation, bias, need_dx, need_dw)


def _run_gated_backward(stream, dh, x, w_gate, w_up, g, u, activation, bias, need_dx, need_dw):
    act = _activation(activation)
    m, k, dtype, device = _first(x, "x")
    n = _rows(w_gate, "w_gate")
    dx = torch.empty((m, k), dtype=x.dtype, device=device) if need_dx else None
    dwg, dwu = (torch.empty((n, k), dtype=x.dtype, device=device) if need_dw else None for _ in range(2))
    dbg, dbu = (torch.empty(n, dtype=x.dtype, device=device) if bias else None for _ in range(2))
    a = _GatedGrad(m, n, k, dtype, act, *_matrix(dh, "dh", m, n, x), *_matrix(x, "x", m, k, x),
                   *_matrix(w_gate, "w_gate", n, k, x), *_matrix(w_up, "w_up", n, k, x), *_matrix(g, "g", m, n, x),
                   *_matrix(u, "u", m, n, x), *((dx.data_ptr(), k) if need_dx else (None, 0)),
                   *((dwg.data_ptr(), k, dwu.data_ptr(), k) if need_dw else (None, 0, None, 0)),
                   *((dbg.data_ptr(), dbu.data_ptr()) if bias else (None, None)))
    _gated_backward(a, device, stream)
    return dx, dwg, dwu, dbg, dbu
