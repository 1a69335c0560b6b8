"""Python binding of the dense layers (include/embx_dense.h): argument marshalling only.

    y = linear(x, weight, bias, residual, activation="relu")
    dx, dw, db = linear_backward(dy, x, weight, z, activation="relu")
    h = gated_ffn(x, w_gate, w_up, b_gate, b_up, activation="silu")
    dx, dw_gate, dw_up, db_gate, db_up = gated_ffn_backward(dh, x, w_gate, w_up, g, u)

Matrices are 2-D device tensors whose rows are contiguous (any row stride of at least a row),
vectors contiguous 1-D ones, all of one dtype: float32, float16 or bfloat16.  Results are
allocated (torch's allocator) unless ``out`` is given; calls run on ``stream`` (a
torch.cuda.Stream or a raw handle), the current stream by default.

The calls are not differentiated by torch: tensors that require a gradient are refused where
gradients are recorded.  Call them under torch.no_grad(), or in forward and backward of a
torch.autograd.Function (``linear`` and ``linear_backward``, say).
"""
from __future__ import annotations

import ctypes

import torch

from . import EmbxError, _lib

try:
    from . import _dense
except ImportError as e:
    raise ImportError(f"embx dense-layer binding missing or not built for this torch ({e}); "
                      "build it with: python paper_2507_01676_amd/build.py") from e

ACTIVATIONS = {"none": 0, "relu": 1, "sigmoid": 2, "silu": 3, "gelu": 4}
_CALLS = ("emb_linear", "emb_linear_backward", "emb_gated", "emb_gated_backward")
_dense.bind(tuple(ctypes.cast(getattr(_lib, name + suffix), ctypes.c_void_p).value for name in _CALLS
                  for suffix in ("", "_workspace")), EmbxError, ACTIVATIONS)


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
    return _dense.linear(x, weight, bias, residual, activation, out, save)


def linear_backward(dy, x, weight, z=None, *, activation="none", bias=True, stream=None, need_dx=True, need_dw=True):
    """Gradients (dx, dweight, dbias) of linear at the gradient dy of its result (None where
    not wanted); z as linear(..., save=True) returned it (not needed with activation
    "none").  The residual's gradient is dy."""
    if stream is not None:
        return _on(stream, linear_backward, dy, x, weight, z, activation=activation, bias=bias, need_dx=need_dx,
                   need_dw=need_dw)
    return _dense.linear_backward(dy, x, weight, z, activation, bias, need_dx, need_dw)


def gated_ffn(x, w_gate, w_up, b_gate=None, b_up=None, *, activation="silu", out=None, save=False, stream=None):
    """act(x w_gate^T + b_gate) * (x w_up^T + b_up) (emb_gated).  x [m, k], weights [n, k],
    biases [n]; ``save``: returns (h, g, u) with both projections, as gated_ffn_backward takes them."""
    if stream is not None:
        return _on(stream, gated_ffn, x, w_gate, w_up, b_gate, b_up, activation=activation, out=out, save=save)
    return _dense.gated(x, w_gate, w_up, b_gate, b_up, activation, out, save)


def gated_ffn_backward(dh, x, w_gate, w_up, g, u, *, activation="silu", bias=False, stream=None, need_dx=True,
                       need_dw=True):
    """Gradients (dx, dw_gate, dw_up, db_gate, db_up) of gated_ffn at the gradient dh of its
    result (None where not wanted); g and u as gated_ffn(..., save=True) returned them."""
    if stream is not None:
        return _on(stream, gated_ffn_backward, dh, x, w_gate, w_up, g, u, activation=activation, bias=bias, need_dx=need_dx,
                   need_dw=need_dw)
    return _dense.gated_backward(dh, x, w_gate, w_up, g, u, activation, bias, need_dx, need_dw)
