"""The serving forms in 64 bits on the host, straight from their formulas, with bounds of the error that
include/embx_serving.h allows.

Bounds.  Quantizing has none: scales and whole numbers are defined exactly.  linear_int8: the sum is a whole number; its
conversion to f32, both scales and the bias are four roundings of 2^-24 of the magnitudes; activation, residual and
result as in dense_reference.  moe: projections as in dense_reference (a scale of 8-bit weights one rounding more), h
rounded to the type; a share exp(l_e - l_0) / total has the rounding of the difference (2^-24 of it) in both exponentials
and the total, and two units of each exponential, n additions and a division; a row's uses are added up in any order."""
from __future__ import annotations

import torch

import dense_reference as R

d = R.d


def quantize(x):
    """(q, scale) as float64"""
    x = d(x)
    largest = x.abs().amax(1) if x.shape[1] else torch.zeros(x.shape[0], dtype=torch.float64)
    fine = torch.isfinite(largest)
    s = torch.where(fine, largest / 127, torch.ones_like(largest)).float().clamp(min=2.0 ** -126).double()
    # (a double's quotient of two floats is a border exactly where the quotient is)
    q = torch.where(fine[:, None], torch.round(torch.where(fine[:, None], x, torch.zeros_like(x)) / s[:, None]).clamp(-127, 127),
                    torch.zeros_like(x))
    return q, torch.where(fine, s, torch.full_like(s, float("nan")))


def linear_int8(q, xs, w, ws, b, r, name, dtype):
    """(y, bound)"""
    q, xs, w, ws, b, r = d(q), d(xs), d(w), d(ws), d(b), d(r)
    z = (q @ w.t()) * xs[:, None] * ws
    ez = 4 * R.SUM * (z.abs() + (0 if b is None else b.abs()))
    if b is not None:
        z = z + b
    y = R.act(z, name)
    ey = R.STEEP * ez + (0 if name in ("none", "relu") else R.FUNC) * (y.abs() + ez)
    if r is not None:
        y, ey = y + r, ey + R.SUM * (y.abs() + r.abs())
    return y, R.rounded(y, ey, dtype)


def route(x, router, top_k, renormalize=True):
    """(chosen, shares, relative bound of the shares)"""
    # (row by row: a matrix product may sum equal rows of the router in different orders, and ties would not be ties)
    logits = torch.stack([(row * d(router)).sum(1) for row in d(x)])
    order = torch.where(torch.isnan(logits), torch.full_like(logits, float("inf")), logits)
    # a stable sort: ties to the lowest; NaN first of all
    chosen = torch.sort(order + 0.0, dim=1, descending=True, stable=True)[1]
    if torch.isnan(logits).any():
        rows = [sorted(range(logits.shape[1]), key=lambda e, i=i: (not bool(torch.isnan(logits[i, e])), -float(order[i, e]), e))
                for i in range(logits.shape[0])]
        chosen = torch.tensor(rows)
    chosen = chosen[:, :top_k]
    far = logits - logits.gather(1, chosen[:, :1])
    e = torch.exp(far)
    kept = e.gather(1, chosen)
    total = (kept if renormalize else e).sum(1, keepdim=True)
    share = kept / total
    n = top_k if renormalize else logits.shape[1]
    spread = far.abs().gather(1, chosen)
    mean = ((kept if renormalize else e) * (spread if renormalize else far.abs())).nan_to_num(0.0).sum(1, keepdim=True) / total
    return chosen, share, (spread + mean + 10 + n) * R.SUM


def moe(x, router, w_gate, w_up, w_down, top_k, name, dtype, scales=None, renormalize=True):
    """((y, bound), chosen, (shares, bound))"""
    chosen, share, eshare = route(x, router, top_k, renormalize)
    x = d(x)
    ws = [d(w) for w in (w_gate, w_up, w_down)]
    more = 0.0
    if scales is not None:
        ws = [w * d(s)[..., None] for w, s in zip(ws, scales)]
        more = 2 * R.SUM
    y, ey, mag = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x)
    for e in range(router.shape[0]):
        rows, places = (chosen == e).nonzero(as_tuple=True)
        if not len(rows):
            continue
        wg, wu, wd = (w[e] for w in ws)
        part = x[rows]
        g, eg = R.affine(part, wg, None)
        u, eu = R.affine(part, wu, None)
        eg, eu = eg + more * g.abs(), eu + more * u.abs()
        a = R.act(g, name)
        ea = R.STEEP * eg + R.FUNC * (a.abs() + eg)
        h = a * u
        eh = ea * (u.abs() + eu) + a.abs() * eu + R.SUM * h.abs()
        if dtype != "f32":
            eh = R.rounded(h, eh, dtype)
        o, bound = h @ wd.t(), eh @ wd.abs().t() + (h.shape[1] + 2) * R.SUM * ((h.abs() + eh) @ wd.abs().t())
        bound = bound + more * o.abs()
        c, ec = share[rows, places][:, None], eshare[rows, places][:, None]
        y[rows] += c * o
        ey[rows] += c * (bound + ec * (o.abs() + bound))
        mag[rows] += c * (o.abs() + bound)
    ey = ey + (top_k + 10) * R.SUM * mag
    return (y, R.rounded(y, ey, dtype)), chosen.int(), (share, share * eshare + R.TINY["f32"])
