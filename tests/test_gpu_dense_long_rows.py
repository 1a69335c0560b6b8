"""The dense layers on rows longer than the 32-bit offsets within a tile reach: millions of inputs, or of outputs in the
gradients.  Operands are -1, 0 and 1, so that every sum is a whole number below 2^24, exact in 32 bits in any order: results
are equal to the products of the same numbers, not near them."""
import pytest

from dense_reference import TYPES
from gpu_helpers import log

pytestmark = pytest.mark.gpu


def units(gen, dtype, *shape):
    import torch
    return torch.randint(-1, 2, shape, generator=gen, dtype=torch.int8, device="cuda").to(TYPES[dtype])


def generator(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def same(got, want, what):
    import torch
    want = want.to(got.dtype)
    if not torch.equal(got, want):
        wrong = (got != want).nonzero()
        rows = sorted(set(wrong[:, 0].tolist()))[:8]
        raise AssertionError(f"{what}: {len(wrong)} of {want.numel()} elements differ, rows {rows}")


# the last: rows that are also copied for their alignment
@pytest.mark.parametrize("dtype,m,n,k", [("f32", 256, 256, 2200000), ("bf16", 512, 260, 5000000), ("f16", 300, 136, 4300001)],
                         ids=str)
def test_many_inputs(gpu_lib, dtype, m, n, k):
    import torch
    log(f"many inputs {dtype} {m} {n} {k}")
    gen = generator(1)
    x, w = units(gen, dtype, m, k), units(gen, dtype, n, k)
    b, r = units(gen, dtype, n), units(gen, dtype, m, n)
    want = x.float() @ w.float().t() + b.float()
    y, z = gpu_lib.linear(x, w, b, r, activation="relu", save=True)
    same(z, want, "z")
    same(y, want.clamp(min=0) + r.float(), "y")
    if dtype == "f32":   # an infinity: the tile with it is computed again
        x[250, k - 3] = float("inf")
        w[:, k - 3] = 1.0
        got = gpu_lib.linear(x, w)
        assert bool(torch.isinf(got[250]).all()) and int((~torch.isfinite(got)).sum()) == n
        x[250, k - 3] = 0.0
        want = x.float() @ w.float().t()
        keep = torch.arange(m, device="cuda") != 250
        same(got[keep], want[keep], "rows beside the infinity")


@pytest.mark.parametrize("dtype,m,n,k", [("f32", 260, 130, 2200000), ("bf16", 300, 200, 4300000)], ids=str)
def test_many_inputs_gated(gpu_lib, dtype, m, n, k):
    log(f"many inputs, gated {dtype} {m} {n} {k}")
    gen = generator(2)
    x, wg, wu = units(gen, dtype, m, k), units(gen, dtype, n, k), units(gen, dtype, n, k)
    _, g, u = gpu_lib.gated_ffn(x, wg, wu, activation="relu", save=True)
    same(g, x.float() @ wg.float().t(), "g")
    same(u, x.float() @ wu.float().t(), "u")


@pytest.mark.parametrize("dtype,m,n,k", [("f32", 512, 2200000, 64), ("bf16", 256, 9000000, 40), ("f16", 200, 5000001, 48),
                                         ("f16", 300, 200, 5000000)], ids=str)
def test_gradients(gpu_lib, dtype, m, n, k):
    log(f"gradients {dtype} {m} {n} {k}")
    gen = generator(3)
    x, w, dy, z = units(gen, dtype, m, k), units(gen, dtype, n, k), units(gen, dtype, m, n), units(gen, dtype, m, n)
    for act in ("relu", "none"):
        dx, dw, db = gpu_lib.linear_backward(dy, x, w, z if act == "relu" else None, activation=act)
        dz = dy.float() * (z > 0) if act == "relu" else dy.float()
        same(dx, dz @ w.float(), f"dx {act}")
        same(dw, dz.t() @ x.float(), f"dw {act}")
        same(db.view(1, -1), dz.sum(0).view(1, -1), f"db {act}")
        del dx, dw, db, dz


@pytest.mark.parametrize("dtype,m,n,k", [("f32", 258, 2200000, 72), ("bf16", 257, 4300003, 64)], ids=str)
def test_gradients_gated(gpu_lib, dtype, m, n, k):
    log(f"gradients, gated {dtype} {m} {n} {k}")
    gen = generator(4)
    x, wg, wu = units(gen, dtype, m, k), units(gen, dtype, n, k), units(gen, dtype, n, k)
    dh, g, u = units(gen, dtype, m, n), units(gen, dtype, m, n), units(gen, dtype, m, n)
    dx, dwg, dwu, dbg, dbu = gpu_lib.gated_ffn_backward(dh, x, wg, wu, g, u, activation="relu", bias=True)
    dg, du = dh.float() * u.float() * (g > 0), dh.float() * g.float().clamp(min=0)
    same(dx, dg @ wg.float() + du @ wu.float(), "dx")
    same(dwg, dg.t() @ x.float(), "dwg")
    same(dwu, du.t() @ x.float(), "dwu")
    same(dbg.view(1, -1), dg.sum(0).view(1, -1), "dbg")
    same(dbu.view(1, -1), du.sum(0).view(1, -1), "dbu")


def test_an_infinite_gradient(gpu_lib):
    """f32: the tiles that it reaches are computed again, from panels too."""
    import torch
    m, n, k = 512, 2200000, 64
    log(f"infinite gradient {m} {n} {k}")
    gen = generator(5)
    x, w, dy = units(gen, "f32", m, k), units(gen, "f32", n, k), units(gen, "f32", m, n)
    x[300], w[n - 5] = 1.0, 1.0
    dy[300, n - 5] = 0.0
    want = [dy @ w, dy.t() @ x]
    dy[300, n - 5] = float("inf")
    dx, dw, db = gpu_lib.linear_backward(dy, x, w)
    for got, value, row in ((dx, want[0], 300), (dw, want[1], n - 5)):
        assert bool(torch.isinf(got[row]).all())
        value[row] = float("inf")
        same(got, value, "dx, dw")
    assert int((~torch.isfinite(db)).sum()) == 1 and bool(torch.isinf(db[n - 5]))
