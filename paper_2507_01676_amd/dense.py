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
import struct

import torch

from . import ERR_INVALID_ARGUMENT, OK, EmbxError, _i32, _lib, _sz, _vp

ACTIVATIONS = {"none": 0, "relu": 1, "sigmoid": 2, "silu": 3, "gelu": 4}
_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
# without the checks of torch's own wrappers, where this torch has them: half a microsecond of a call
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)


class _Entry:
    """A call of the library and its struct.  The struct's fields are packed as the header lists them: m, n, k, dtype,
    activation, then matrices (pointer, row stride; "M") and vectors (pointer; "V").  (A small call's time is the
    host's: a ctypes.Structure takes three times as long to fill.)"""

    def __init__(self, name, layout, asks):
        self.name = name
        self.asks = asks   # most calls need a workspace: its size is asked for first, not after a refusal
        packer = struct.Struct("@qqqii" + "".join("Pq" if f == "M" else "P" for f in layout))
        self.pack, self.bytes = packer.pack, packer.size
        self.fn, self.size = getattr(_lib, name), getattr(_lib, name + "_workspace")
        self.fn.restype, self.fn.argtypes = _i32, [ctypes.c_char_p, _vp, _sz, _vp]
        self.size.restype, self.size.argtypes = _i32, [ctypes.c_char_p, ctypes.POINTER(_sz)]

    def __call__(self, a, x, device):
        stream = _current_stream(device)
        code = ERR_INVALID_ARGUMENT if self.asks else self.fn(a, None, 0, stream)
        if code == ERR_INVALID_ARGUMENT:
            nbytes = _sz(0)
            code = self.size(a, nbytes)
            if code == OK:
                nbytes = nbytes.value
                ws = x.new_empty(nbytes, dtype=torch.uint8)
                code = self.fn(a, ws.data_ptr(), nbytes, stream)
        if code != OK:
            raise EmbxError(code, self.name)


_linear = _Entry("emb_linear", "MMVMMM", False)                  # x weight bias residual y z
_linear_backward = _Entry("emb_linear_backward", "MMMMMMV", True)   # dy x weight z dx dweight dbias
_gated = _Entry("emb_gated", "MMMVVMMM", False)                  # x w_gate w_up b_gate b_up h g u
_gated_backward = _Entry("emb_gated_backward", "MMMMMMMMMVV", True)   # dh x w_gate w_up g u dx dw_gate dw_up db_gate db_up
_NONE = (0, 0)


def _activation(name) -> int:
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}, got {name!r}") from None


def _first(x, name):
    """(rows, columns, dtype, its code, device index, (pointer, row stride)) of the matrix that the others are measured
    against."""
    try:
        rows, cols = x.shape
        dtype, device = x.dtype, x.get_device()
        code = _DTYPES[dtype]
        if device >= 0 and device == _current_device():
            ld, step = x.stride()
            at = (x.data_ptr(), ld) if step == 1 and ld >= cols else _odd_matrix(x, name, rows, cols, dtype, device)
            return rows, cols, dtype, code, device, at
    except (AttributeError, KeyError, TypeError):
        pass
    except ValueError:
        if isinstance(x, torch.Tensor) and x.dim() == 2:
            raise
    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dim() == 2):
        raise ValueError(f"{name} must be a 2-D device tensor")
    if x.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32, float16 or bfloat16, got {x.dtype}")
    raise ValueError(f"{name} is on cuda:{x.get_device()}, the current device is cuda:{_current_device()}")


def _matrix(t, name, rows, cols, dtype, device):
    """(pointer, row stride) of a matrix [rows, cols]."""
    try:
        if t.dtype is dtype and t.get_device() == device and t.shape == (rows, cols):
            ld, step = t.stride()
            if step == 1 and ld >= cols:
                return t.data_ptr(), ld
    except AttributeError:
        pass
    return _odd_matrix(t, name, rows, cols, dtype, device)


def _odd_matrix(t, name, rows, cols, dtype, device):
    """The same of a matrix of one row or column with other strides; says what is wrong with any other."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.get_device() == device and t.dim() == 2):
        raise ValueError(f"{name} must be a 2-D {dtype} tensor on cuda:{device}")
    r, c = t.shape
    if r != rows or c != cols:
        raise ValueError(f"{name} must be [{rows}, {cols}], got {list(t.shape)}")
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{name} must have contiguous rows, got strides {t.stride()}")
    if ld < cols:
        if rows > 1:
            raise ValueError(f"{name}: rows must not overlap, got strides {t.stride()}")
        ld = cols
    return t.data_ptr(), ld


def _rows(t, name):
    if not (isinstance(t, torch.Tensor) and t.dim() == 2):
        raise ValueError(f"{name} must be a 2-D device tensor")
    return t.shape[0]


def _vector(t, name, n, dtype, device):
    if t is None:
        return 0
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device and t.shape == (n,)
            and (t.stride() == (1,) or n == 1)):
        raise ValueError(f"{name} must be a contiguous [{n}] {dtype} tensor on cuda:{device}")
    return t.data_ptr()


def _on(stream, fn, *args, **options):
    """fn(...) with the launches and torch's allocations on that stream."""
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    with torch.cuda.stream(stream):
        return fn(*args, **options)


def linear(x, weight, bias=None, residual=None, *, activation="none", out=None, save=False, stream=None):
    """act(x weight^T + bias) + residual (emb_linear).  x [m, k], weight [n, k], bias [n],
    residual [m, n]; ``save``: also returns the sums before the activation, as
    linear_backward takes them.  ``out`` may be the residual."""
    if stream is not None:
        return _on(stream, linear, x, weight, bias, residual, activation=activation, out=out, save=save)
    act = _activation(activation)
    m, k, dtype, code, device, at = _first(x, "x")
    n = _rows(weight, "weight")
    y = x.new_empty(m, n) if out is None else out
    z = x.new_empty(m, n) if save else None
    _linear(_linear.pack(m, n, k, code, act, *at,
                         *_matrix(weight, "weight", n, k, dtype, device), _vector(bias, "bias", n, dtype, device),
                         *(_NONE if residual is None else _matrix(residual, "residual", m, n, dtype, device)),
                         *((y.data_ptr(), n) if out is None else _matrix(y, "out", m, n, dtype, device)),
                         *((z.data_ptr(), n) if save else _NONE)), x, device)
    return (y, z) if save else y


def linear_backward(dy, x, weight, z=None, *, activation="none", bias=True, stream=None, need_dx=True, need_dw=True):
    """Gradients (dx, dweight, dbias) of linear at the gradient dy of its result (None where
    not wanted); z as linear(..., save=True) returned it (not needed with activation
    "none").  The residual's gradient is dy."""
    if stream is not None:
        return _on(stream, linear_backward, dy, x, weight, z, activation=activation, bias=bias, need_dx=need_dx,
                   need_dw=need_dw)
    act = _activation(activation)
    m, k, dtype, code, device, at = _first(x, "x")
    n = _rows(weight, "weight")
    if act and z is None:
        raise ValueError(f"activation {activation!r} needs z, the sums that linear(..., save=True) returns")
    dx = x.new_empty(m, k) if need_dx else None
    dw = x.new_empty(n, k) if need_dw else None
    db = x.new_empty(n) if bias else None
    _linear_backward(_linear_backward.pack(
        m, n, k, code, act, *_matrix(dy, "dy", m, n, dtype, device), *at,
        *_matrix(weight, "weight", n, k, dtype, device), *(_matrix(z, "z", m, n, dtype, device) if act else _NONE),
        *((dx.data_ptr(), k) if need_dx else _NONE), *((dw.data_ptr(), k) if need_dw else _NONE),
        db.data_ptr() if bias else 0), x, device)
    return dx, dw, db


def gated_ffn(x, w_gate, w_up, b_gate=None, b_up=None, *, activation="silu", out=None, save=False, stream=None):
    """act(x w_gate^T + b_gate) * (x w_up^T + b_up) (emb_gated).  x [m, k], weights [n, k],
    biases [n]; ``save``: returns (h, g, u) with both projections, as gated_ffn_backward takes them."""
    if stream is not None:
        return _on(stream, gated_ffn, x, w_gate, w_up, b_gate, b_up, activation=activation, out=out, save=save)
    act = _activation(activation)
    m, k, dtype, code, device, at = _first(x, "x")
    n = _rows(w_gate, "w_gate")
    h = x.new_empty(m, n) if out is None else out
    g, u = ((x.new_empty(m, n), x.new_empty(m, n)) if save else (None, None))
    _gated(_gated.pack(m, n, k, code, act, *at,
                       *_matrix(w_gate, "w_gate", n, k, dtype, device), *_matrix(w_up, "w_up", n, k, dtype, device),
                       _vector(b_gate, "b_gate", n, dtype, device), _vector(b_up, "b_up", n, dtype, device),
                       *((h.data_ptr(), n) if out is None else _matrix(h, "out", m, n, dtype, device)),
                       *((g.data_ptr(), n, u.data_ptr(), n) if save else (0, 0, 0, 0))), x, device)
    return (h, g, u) if save else h


def gated_ffn_backward(dh, x, w_gate, w_up, g, u, *, activation="silu", bias=False, stream=None, need_dx=True,
                       need_dw=True):
    """Gradients (dx, dw_gate, dw_up, db_gate, db_up) of gated_ffn at the gradient dh of its
    result (None where not wanted); g and u as gated_ffn(..., save=True) returned them."""
    if stream is not None:
        return _on(stream, gated_ffn_backward, dh, x, w_gate, w_up, g, u, activation=activation, bias=bias, need_dx=need_dx,
                   need_dw=need_dw)
    act = _activation(activation)
    m, k, dtype, code, device, at = _first(x, "x")
    n = _rows(w_gate, "w_gate")
    dx = x.new_empty(m, k) if need_dx else None
    dwg, dwu = ((x.new_empty(n, k), x.new_empty(n, k)) if need_dw else (None, None))
    dbg, dbu = ((x.new_empty(n), x.new_empty(n)) if bias else (None, None))
    _gated_backward(_gated_backward.pack(
        m, n, k, code, act, *_matrix(dh, "dh", m, n, dtype, device), *at,
        *_matrix(w_gate, "w_gate", n, k, dtype, device), *_matrix(w_up, "w_up", n, k, dtype, device),
        *_matrix(g, "g", m, n, dtype, device), *_matrix(u, "u", m, n, dtype, device),
        *((dx.data_ptr(), k) if need_dx else _NONE),
        *((dwg.data_ptr(), k, dwu.data_ptr(), k) if need_dw else (0, 0, 0, 0)),
        *((dbg.data_ptr(), dbu.data_ptr()) if bias else (0, 0))), x, device)
    return dx, dwg, dwu, dbg, dbu
