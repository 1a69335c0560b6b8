"""The dense layers in 64 bits on the host, straight from their formulas, with bounds of the error that
a sum in 32 bits and the roundings named in include/embx_dense.h may make.

Bounds.  A sum of n products formed in 32 bits, in any order, is off by at most (n + 2) 2^-24 times the
sum of the products' magnitudes.  An activation or slope computed in 32 bits adds at most 2^-20 of its
magnitude (a few roundings of exp, erf and a reciprocal) and passes an error of its argument on with its
steepest slope, at most 1.13 (slopes: 1 at most).  A result rounded to its type is off by half a unit in
the last place: 2^-24, 2^-11 or 2^-8 of its magnitude, or less than the smallest number of the type."""
from __future__ import annotations

import math

import torch

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # bf16: 8 significant bits
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}
SUM = 2.0 ** -24
FUNC = 2.0 ** -20
STEEP = 1.13


def act(z, name):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "sigmoid":
        return torch.sigmoid(z)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "sigmoid":
        return torch.sigmoid(z) * torch.sigmoid(-z)
    if name == "silu":
        return torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    if name == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def d(t):
    return None if t is None else t.detach().double().cpu()


def rounded(value, error, dtype):
    """Bound of |result - value| where the result is a 32-bit value within error, rounded to dtype."""
    return error + ROUND[dtype] * (value.abs() + error) + TINY[dtype]


def affine(x, w, b):
    z, mag = x @ w.t(), x.abs() @ w.abs().t()
    if b is not None:
        z, mag = z + b, mag + b.abs()
    return z, (x.shape[1] + 2) * SUM * mag


def linear(x, w, b, r, name, dtype):
    """((y, bound), (z, bound))"""
    x, w, b, r = d(x), d(w), d(b), d(r)
    z, ez = affine(x, w, b)
    y = act(z, name)
    ey = STEEP * ez + (0 if name in ("none", "relu") else FUNC) * (y.abs() + ez)
    if r is not None:
        y, ey = y + r, ey + SUM * (y.abs() + r.abs())
    return (y, rounded(y, ey, dtype)), (z, rounded(z, ez, dtype))


def gated(x, wg, wu, bg, bu, name, dtype):
    """((h, bound), (g, bound), (u, bound))"""
    x, wg, wu, bg, bu = d(x), d(wg), d(wu), d(bg), d(bu)
    g, eg = affine(x, wg, bg)
    u, eu = affine(x, wu, bu)
    a = act(g, name)
    ea = STEEP * eg + FUNC * (a.abs() + eg)
    h = a * u
    eh = ea * (u.abs() + eu) + a.abs() * eu + SUM * h.abs()
    return (h, rounded(h, eh, dtype)), (g, rounded(g, eg, dtype)), (u, rounded(u, eu, dtype))


def _products(dzs, edzs, ws, x, dtype):
    """dx = sum of dz W, dW = dz^T x each, db = column sums each, with bounds; dz is rounded to dtype
    before the products (not before the column sums)."""
    m, k = x.shape
    n = dzs[0].shape[1]
    dx, edx = torch.zeros(m, k, dtype=torch.float64), torch.zeros(m, k, dtype=torch.float64)
    dws, dbs = [], []
    half = 0.0 if dtype == "f32" else 1.0
    for dz, edz, w in zip(dzs, edzs, ws):
        e = edz + half * (ROUND[dtype] * (dz.abs() + edz) + TINY[dtype])
        dx = dx + dz @ w
        edx = edx + e @ w.abs() + (2 * n + 2) * SUM * ((dz.abs() + e) @ w.abs())
        ew = e.t() @ x.abs() + (m + 2) * SUM * ((dz.abs() + e).t() @ x.abs())
        dw = dz.t() @ x
        dws.append((dw, rounded(dw, ew, dtype)))
        db = dz.sum(0)
        dbs.append((db, rounded(db, edz.sum(0) + (m + 2) * SUM * (dz.abs() + edz).sum(0), dtype)))
    return [(dx, rounded(dx, edx, dtype)), *dws, *dbs]


def linear_backward(dy, x, w, z, name, dtype):
    """[(dx, bound), (dw, bound), (db, bound)]"""
    dy, x, w = d(dy), d(x), d(w)
    if name == "none":
        return _products([dy], [torch.zeros_like(dy)], [w], x, dtype) if dtype == "f32" else \
            _exact_products(dy, x, w, dtype)
    s = slope(d(z), name)
    dz = dy * s
    edz = (0.0 if name == "relu" else FUNC) * dy.abs() * (s.abs() + 1)
    return _products([dz], [edz], [w], x, dtype)


def _exact_products(dy, x, w, dtype):
    """Without an activation dz is dy itself: nothing is rounded before the products."""
    m, k = x.shape
    n = dy.shape[1]
    dx, dw, db = dy @ w, dy.t() @ x, dy.sum(0)
    return [(dx, rounded(dx, (n + 2) * SUM * (dy.abs() @ w.abs()), dtype)),
            (dw, rounded(dw, (m + 2) * SUM * (dy.abs().t() @ x.abs()), dtype)),
            (db, rounded(db, (m + 2) * SUM * dy.abs().sum(0), dtype))]


def gated_backward(dh, x, wg, wu, g, u, name, dtype):
    """[(dx, b), (dwg, b), (dwu, b), (dbg, b), (dbu, b)]"""
    dh, x, wg, wu, g, u = (d(t) for t in (dh, x, wg, wu, g, u))
    s, a = slope(g, name), act(g, name)
    dg, du = dh * u * s, dh * a
    edg = dh.abs() * u.abs() * (FUNC * (s.abs() + 1) + 2 * SUM * s.abs())
    edu = dh.abs() * FUNC * (a.abs() + g.abs())
    return _products([dg, du], [edg, edu], [wg, wu], x, dtype)


def check(got, want, what):
    """got within its bound of (value, bound), element by element; not finite where the value is not."""
    value, bound = want
    got = d(got)
    assert got.shape == value.shape, f"{what}: shape {tuple(got.shape)}, not {tuple(value.shape)}"
    assert torch.equal(torch.isnan(got), torch.isnan(value)), f"{what}: NaN in other places"
    fine = torch.isfinite(value)
    assert torch.equal(got[~fine & ~torch.isnan(value)], value[~fine & ~torch.isnan(value)]), f"{what}: infinities differ"
    off = (got - value).abs()[fine] - bound[fine]
    assert off.numel() == 0 or off.max() <= 0, \
        f"{what}: {int((off > 0).sum())} of {off.numel()} elements out of bounds, worst by {off.max():.3g}"
