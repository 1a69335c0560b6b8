"""The layer of experts in 64 bits on the host, with the error that include/embx_serving.h allows where act(..) * (..) goes into
the product with Wd in 32 bits, and operands that show fewer.

Bounds.  As in serving_reference, but act(..) * (..), h, is not rounded to the layer's type.  Weights of f16 multiply it as two
f16 values of it times a power of two: 2^-23 of it, or 2^-36 of its row's largest.  A sum of products of which some are nought is
off by the others only: of two in 16 bits or none, not at all but where they are added (their product has 22 bits at most), of n
at most (n + 2) 2^-24 times the magnitudes; the down projection adds up to three values for each h."""
from __future__ import annotations

import torch

import dense_reference as R
import serving_reference as S

d = R.d


def moe(x, router, w_gate, w_up, w_down, top_k, name, dtype, scales=None, renormalize=True, handed=None):
    """((y, bound), chosen, (shares, bound)).  ``handed``: what h is replaced by before the product with Wd, a function of h
    and Wd that gives both."""
    chosen, share, eshare = S.route(x, router, top_k, renormalize)
    x = d(x)
    ws = [d(w) for w in (w_gate, w_up, w_down)]
    more = 0.0
    if scales is not None:
        ws = [w * d(s)[..., None] for w, s in zip(ws, scales)]
        more = 2 * R.SUM
    y, ey, mag = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x)

    def project(part, w):
        count = (part != 0).double() @ (w != 0).double().t()
        z = part @ w.t()
        own = torch.where(count > (0 if dtype == "f32" else 1), count + 2, torch.zeros_like(count)) * R.SUM
        return z, (own + more) * (part.abs() @ w.abs().t())

    for e in range(router.shape[0]):
        rows, places = (chosen == e).nonzero(as_tuple=True)
        if not len(rows):
            continue
        wg, wu, wd = (w[e] for w in ws)
        g, eg = project(x[rows], wg)
        u, eu = project(x[rows], wu)
        a = R.act(g, name)
        ea = R.STEEP * eg + (0 if name in ("none", "relu") else R.FUNC) * (a.abs() + eg)
        h = a * u
        eh = ea * (u.abs() + eu) + a.abs() * eu + R.SUM * h.abs()
        if handed is not None:
            h, wd = handed(h.float(), wd.float())
            h, wd = h.double(), wd.double()
        elif dtype == "f16" and scales is None:
            eh = eh + 2.0 ** -23 * (h.abs() + eh) + 2.0 ** -36 * h.abs().amax(1, keepdim=True)
        used = (h != 0).double() @ (wd != 0).double().t()
        o, bound = h @ wd.t(), eh @ wd.abs().t() + (3 * used + 2) * R.SUM * ((h.abs() + eh) @ wd.abs().t())
        bound = bound + more * o.abs()
        c, ec = share[rows, places][:, None], eshare[rows, places][:, None]
        y[rows] += c * o
        ey[rows] += c * (bound + ec * (o.abs() + bound))
        mag[rows] += c * (o.abs() + bound)
    ey = ey + (top_k + 10) * R.SUM * mag
    return (y, R.rounded(y, ey, dtype)), chosen.int(), (share, share * eshare + R.TINY["f32"])


SPREADS = ["even", "small", "large", "mixed"]


def operands(size, dtype, seed, eight, spread="even", device="cpu"):
    """Operands whose results are differences of two nearly equal h: bits of h that are left out show.  A row of x has two values
    that are not nought; h of each odd column differs from the one before by 2^-11 or so of itself, and an output is the
    difference of one such pair.  ``spread``: h about one; about 2^-20; about 2^20; or of all sizes between.  Returns a dict of
    x, router, ws, scales and top_k."""
    m, f, dim, e, top = size
    gen = torch.Generator().manual_seed(seed)
    t = R.TYPES[dtype]

    def uniform(*shape):
        return 1.0 + torch.rand(*shape, generator=gen, dtype=torch.float64)

    def signs(*shape):
        return 1.0 - 2.0 * torch.randint(0, 2, shape, generator=gen).double()

    x = torch.zeros(m, dim, dtype=torch.float64)
    first, second = torch.randperm(dim, generator=gen)[[0, -1]].tolist()
    x[:, second] = uniform(m) * 2.0 ** -13
    x[:, first] = uniform(m)
    router = torch.randn(e, dim, generator=gen, dtype=torch.float64)
    pairs = f // 2

    def twice(w):   # (a last column of no pair is nought)
        return torch.cat([w.repeat_interleave(2, 1), w.new_zeros(e, f % 2, *w.shape[2:])], 1)

    power = {"even": torch.zeros(e, pairs), "small": torch.full((e, pairs), -10.0), "large": torch.full((e, pairs), 10.0),
             "mixed": torch.round(torch.linspace(-10, 10, max(pairs, 1))[:pairs].repeat(e, 1) * signs(e, 1))}[spread].double()
    gate, up = uniform(e, pairs, dim) * signs(e, pairs, dim), uniform(e, pairs, dim) * signs(e, pairs, dim)
    scale, down_power = torch.ones(e, pairs, dtype=torch.float64), -torch.round(power * (1.4 if spread == "small" else 0.7))
    if eight:
        gate, up = torch.round(gate * 63), torch.round(up * 63)
        scale = 2.0 ** (power - 6)
    else:
        gate, up = gate * 2.0 ** power[..., None], up * 2.0 ** power[..., None]
    gate, up, scale = twice(gate), twice(up), twice(scale[..., None])[..., 0]
    gate[:, 1::2, second] *= -1.0
    down = torch.zeros(e, dim, f, dtype=torch.float64)
    if pairs:
        at = (torch.arange(dim) + torch.randint(0, pairs, (e, 1), generator=gen)) * max(1, pairs // dim) % pairs
        one = torch.ones(e, dim, dtype=torch.float64) if eight else 2.0 ** down_power.gather(1, at) * uniform(e, dim)
        down.scatter_(2, 2 * at[..., None], one[..., None])
        down.scatter_(2, 2 * at[..., None] + 1, -one[..., None])
    o = dict(x=x.to(t), router=router.to(t), top_k=top, scales=None)
    if eight:
        o["ws"] = [w.to(torch.int8) for w in (gate, up, down)]
        rows = 2.0 ** (down_power.gather(1, at)) if pairs else torch.ones(e, dim)
        o["scales"] = tuple(s.float().to(device) for s in (scale, scale, rows))
    else:
        o["ws"] = [w.to(t) for w in (gate, up, down)]
    o["ws"] = [w.to(device) for w in o["ws"]]
    o["x"], o["router"] = o["x"].to(device), o["router"].to(device)
    return o


def bf16_parts(count):
    """h as `count` bf16 values that are added up"""
    def hand(h, wd):
        left, total = h, torch.zeros_like(h)
        for _ in range(count):
            part = left.bfloat16().float()
            total, left = total + part, left - part
        return total, wd
    return hand


def f16_parts(count):
    """h as `count` f16 values that are added up"""
    def hand(h, wd):
        left, total = h.double(), torch.zeros_like(h, dtype=torch.float64)
        for _ in range(count):
            part = left.to(torch.float16).double()
            total, left = total + part, left - part
            left = torch.where(torch.isfinite(left), left, torch.zeros_like(left))
        return total, wd
    return hand
