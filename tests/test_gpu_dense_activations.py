"""The f32 activations and slopes against 64 bits at given sums, relative to the value itself: also where it is small.

A layer of one input with the weight 1 passes its x on exactly; a gradient of one output with the weight 1 is the slope, off
by 2^-22 of itself more (its product).  Bounds, with u = 2^-23, a unit in the last place at most: exp of the hardware 1 u and
1/2 for the correction of its argument, 1 + t half a u and at most half of t's error, the reciprocal 1, each product 1/2: 5 u
for the sigmoid and z sigmoid(z).  The normal distribution's erfc has an argument that is rounded, as a constant is, and so
is off by 3/4 u of itself, which erfc passes on z^2 + 1 times, and 16 u at most of its own; exp(-z^2 / 2) is off by z^2 / 4 u
for its argument and by 4 u.  Below the normal numbers a unit is 2^-149."""
import math

import pytest

from gpu_helpers import log

pytestmark = pytest.mark.gpu
U, LEAST = 2.0 ** -23, 2.0 ** -149


def sums(top):
    """exact f32 values: evenly spread, around nought, and just above the ends of exp"""
    import torch
    gen = torch.Generator().manual_seed(1)
    z = torch.cat([torch.linspace(-top, top, 20001), torch.randn(5000, generator=gen), torch.randn(2000, generator=gen) * 1e-3,
                   torch.linspace(-min(top, 89.0), -min(top, 87.0), 3001), torch.tensor([0.0, -0.0, 1e-30, -1e-30])])
    return z.float()


def phi(z):
    import torch
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def check(got, want, bound, z):
    off = (got.double().cpu().view(-1) - want).abs()
    at = int((off / bound).argmax())
    assert off[at] <= bound[at], \
        f"z = {z[at].item()!r}: {got.view(-1)[at].item()!r}, not {want[at].item()!r}; {off[at] / bound[at]:.2f} of the bound"


@pytest.mark.parametrize("act,top", [("sigmoid", 100.0), ("silu", 100.0), ("gelu", 12.5)])
def test_values(gpu_lib, act, top):
    import torch
    log(act)
    z = sums(top)
    got = gpu_lib.linear(z.view(-1, 1).cuda(), torch.ones(1, 1, device="cuda"), activation=act)
    d = z.double()
    s = torch.sigmoid(d)
    if act == "sigmoid":
        want, bound = s, 5 * U * s + 2 * LEAST
    elif act == "silu":
        want, bound = d * s, 5 * U * d.abs() * s + 2 * LEAST * (d.abs() + 1)
    else:
        p = phi(d)
        want, bound = d * p, (0.75 * (d * d + 1) + 17) * U * d.abs() * p + 2 * LEAST * (d.abs() + 1)
    check(got, want, bound, z)
    gated = gpu_lib.gated_ffn(z.view(-1, 1).cuda(), torch.ones(1, 1, device="cuda"), torch.zeros(1, 1, device="cuda"), None,
                              torch.ones(1, device="cuda"), activation=act)
    check(gated, want, bound, z)


@pytest.mark.parametrize("act,top", [("sigmoid", 80.0), ("silu", 80.0), ("gelu", 12.0)])
def test_slopes(gpu_lib, act, top):
    import torch
    log(act)
    z = sums(top)
    one = torch.ones(1, 1, device="cuda")
    dx, _, _ = gpu_lib.linear_backward(torch.ones(len(z), 1, device="cuda"), torch.ones(len(z), 1, device="cuda"), one,
                                       z.view(-1, 1).cuda(), activation=act)
    d = z.double()
    s, c = torch.sigmoid(d), torch.sigmoid(-d)
    if act == "sigmoid":
        want = s * c
        size = 8 * U * want
    elif act == "silu":
        want = s * (1 + d * c)
        size = 10 * U * s * (1 + d.abs() * c)
    else:
        p, bell = phi(d), torch.exp(-d * d / 2) / math.sqrt(2 * math.pi)
        want = p + d * bell
        size = U * ((0.75 * (d * d + 1) + 17) * p + (0.25 * d * d + 6) * d.abs() * bell)
    check(dx, want, size + 2.0 ** -22 * want.abs() + 4 * LEAST, z)


@pytest.mark.parametrize("act", ["sigmoid", "silu", "gelu"])
def test_not_finite_and_far_out(gpu_lib, act):
    import torch
    z = torch.tensor([[1e30], [-1e30], [3e38], [-3e38], [128.5], [-128.5], [1000.0], [-1000.0], [float("nan")], [float("inf")]])
    got = gpu_lib.linear(z.cuda(), torch.ones(1, 1, device="cuda"), activation=act).cpu().view(-1)
    up = {"sigmoid": torch.ones(10), "silu": z.view(-1), "gelu": z.view(-1)}[act]
    down = torch.zeros(10)
    want = torch.where(z.view(-1) > 0, up, down)
    assert torch.isnan(got[8])
    got[8] = 0.0
    assert torch.equal(got, want), got
