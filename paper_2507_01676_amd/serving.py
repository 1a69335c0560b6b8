"""Python binding of the dense layers' serving forms (include/embx_serving.h): argument marshalling only.

    q, scale = quantize_rows(weight)                                  # once, when a model is loaded
    y = linear_int8(x, q, scale, bias, residual, activation="relu")   # x's rows are quantized on the way
    y = moe_ffn(x, router, w_gate, w_up, w_down, top_k=2)             # a few of the experts for each row

Matrices are 2-D device tensors whose rows are contiguous (any row stride of at least a row), those of experts 3-D ones
[experts, rows, cols] with contiguous rows, vectors and scales contiguous.  Results are allocated (torch's allocator)
unless ``out`` is given; calls run on ``stream`` (a torch.cuda.Stream or a raw handle), the current stream by default.

The calls have no gradient: tensors that require one are refused where gradients are recorded.
"""
from __future__ import annotations

import ctypes

from . import _lib
from .dense import _dense, _on

_dense.bind_serving(tuple(ctypes.cast(getattr(_lib, name), ctypes.c_void_p).value for name in (
    "emb_quantize", "emb_linear_int8", "emb_linear_int8_workspace", "emb_moe", "emb_moe_workspace")))


def quantize_rows(x, *, out=None, stream=None):
    """(q, scale) of the rows of x [m, k] (emb_quantize): q int8 [m, k] and scale float32 [m], with x about scale * q.
    ``out``: a pair of tensors for both.  Rows of a q that is allocated start at multiples of 16 bytes, as linear_int8
    reads them fastest: its row stride is k rounded up to that."""
    if stream is not None:
        return _on(stream, quantize_rows, x, out=out)
    return _dense.quantize(x, *((None, None) if out is None else out))


def linear_int8(x, weight, w_scale, bias=None, residual=None, *, x_scale=None, activation="none", dtype=None, out=None,
                stream=None):
    """act((x * x_scale) (weight * w_scale)^T + bias) + residual (emb_linear_int8).  weight int8 [n, k], w_scale float32
    [n].  x [m, k]: int8 with ``x_scale`` float32 [m], or float32, float16 or bfloat16 without, whose rows are quantized as
    quantize_rows does.  bias [n], residual and result [m, n] have ``dtype``: x's, if that is not int8; else ``out``'s, the
    residual's or the bias's, or bfloat16.  ``out`` may be the residual."""
    if stream is not None:
        return _on(stream, linear_int8, x, weight, w_scale, bias, residual, x_scale=x_scale, activation=activation, dtype=dtype,
                   out=out)
    return _dense.linear_int8(x, weight, w_scale, bias, residual, x_scale, activation, dtype, out)


def moe_ffn(x, router, w_gate, w_up, w_down, *, top_k, scales=None, activation="silu", renormalize=True, out=None,
            routing=False, stream=None):
    """The layer of experts (emb_moe).  x [m, d], router [experts, d], w_gate and w_up [experts, f, d], w_down
    [experts, d, f], all of x's dtype; or the experts' matrices int8 with ``scales``, float32 [experts, f], [experts, f] and
    [experts, d].  Each row takes the ``top_k`` experts of the largest logits, with shares that are the softmax over those
    (``renormalize``) or over all.  ``routing``: returns (y, experts, shares) with both [m, top_k], int32 and float32."""
    if stream is not None:
        return _on(stream, moe_ffn, x, router, w_gate, w_up, w_down, top_k=top_k, scales=scales, activation=activation,
                   renormalize=renormalize, out=out, routing=routing)
    return _dense.moe(x, router, w_gate, w_up, w_down, top_k, *((None, None, None) if scales is None else scales), activation,
                      renormalize, out, routing)
