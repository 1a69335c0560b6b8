"""Every kernel of the dense layers (the sizes of dense_kernels.py, which test_dense_choice.py holds to their kernels):
results against 64 bits, whole numbers exactly, infinities and NaN in their rows only, operands inside larger matrices,
the result over the residual, and the ends of f32's range on the tiles that take f32 values apart."""
import pytest

import dense_kernels as K
import dense_reference as R
from gpu_helpers import log

pytestmark = pytest.mark.gpu
FORWARD, BACKWARD = K.each(K.FORWARD), K.each(K.BACKWARD)


def normal(gen, dtype, *shape, std=1.0):
    import torch
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(R.TYPES[dtype])


def whole_numbers(gen, dtype, *shape):
    import torch
    return torch.randint(-2, 3, shape, generator=gen, device="cuda").to(R.TYPES[dtype])


def generator(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def operands(make, case, seed):
    """x, weights, biases and residual of a forward case"""
    op, dtype, (m, n, k) = case[:3]
    gen = generator(seed)
    x, r = make(gen, dtype, m, k), make(gen, dtype, m, n)
    ws = [make(gen, dtype, n, k) for _ in range(1 if op == "linear" else 2)]
    return x, ws, [make(gen, dtype, n) for _ in ws], r


def scaled(gen, dtype, *shape):
    # weights [n, k] as k^-1/2, so that sums are of order one whatever the operand's place
    return normal(gen, dtype, *shape, std=1.0 if len(shape) == 1 else shape[1] ** -0.25)


def run(lib, case, x, ws, bs, r, act, **kw):
    """(result, saved sums ..)"""
    if case[0] == "linear":
        return lib.linear(x, ws[0], bs[0], r, activation=act, save=True, **kw)
    return lib.gated_ffn(x, *ws, *bs, activation=act, save=True, **kw)


@pytest.mark.parametrize("case", FORWARD, ids=K.name)
def test_forward(gpu_lib, case):
    log(K.name(case))
    x, ws, bs, r = operands(scaled, case, 1)
    got = run(gpu_lib, case, x, ws, bs, r, "silu")
    if case[0] == "linear":
        want = R.linear(x, ws[0], bs[0], r, "silu", case[1])
    else:
        want = R.gated(x, *ws, *bs, "silu", case[1])
    for g, w, what in zip(got, want, ("result", "saved", "saved u")):
        R.check(g, w, what)


@pytest.mark.parametrize("case", FORWARD, ids=K.name)
def test_whole_numbers(gpu_lib, case):
    """Sums of whole numbers are exact in 32 bits: equal results, also over the residual and from operands inside larger
    matrices (of NaN), outside which nothing is written."""
    import torch
    log(K.name(case))
    op, dtype, (m, n, k) = case[:3]
    x, ws, bs, r = operands(whole_numbers, case, 2)
    sums = [x.float() @ w.float().t() + b.float() for w, b in zip(ws, bs)]
    y = sums[0].clamp(min=0) + r.float() if op == "linear" else sums[0].clamp(min=0) * sums[1]
    want = [t.to(x.dtype) for t in (y, *sums)]
    for g, w, what in zip(run(gpu_lib, case, x, ws, bs, r, "relu"), want, ("result", "saved", "saved u")):
        assert torch.equal(g, w), what
    if op == "linear":
        over = r.clone()
        assert gpu_lib.linear(x, ws[0], bs[0], over, activation="relu", out=over) is over
        assert torch.equal(over, want[0]), "over the residual"
    left = 8 if case[5] else 3

    def inside(t):
        big = torch.full((t.shape[0] + 2, t.shape[1] + left + 8), float("nan"), dtype=t.dtype, device="cuda")
        view = big[1:-1, left:left + t.shape[1]]
        view.copy_(t)
        return view, big

    out, around = inside(torch.zeros_like(r))
    got = run(gpu_lib, case, inside(x)[0], [inside(w)[0] for w in ws], bs, inside(r)[0], "relu", out=out)
    for g, w, what in zip(got, want, ("result", "saved", "saved u")):
        assert torch.equal(g, w), what + " of views"
    around[1:-1, left:left + n] = float("nan")
    assert bool(torch.isnan(around).all()), "written outside the result"


@pytest.mark.parametrize("case", FORWARD, ids=K.name)
def test_not_finite(gpu_lib, case):
    """An infinity, a NaN and (f32) the largest number in rows of x reach those rows' results alone."""
    import torch
    log(K.name(case))
    op, dtype, (m, n, k) = case[:3]
    x, ws, bs, r = operands(scaled, case, 3)
    for t in (x, *ws):
        t[t == 0] = 0.5
    rows = sorted({0, 1, m // 2, m - 2, m - 1})
    x[rows[1], k - 1] = float("inf")
    x[rows[-1], k // 2] = float("nan")
    x[rows[2], 0] = float("-inf")
    got = run(gpu_lib, case, x, ws, bs, r, "none")
    part = x[rows]
    if op == "linear":
        want = R.linear(part, ws[0], bs[0], r[rows], "none", dtype)
    else:
        want = R.gated(part, *ws, *bs, "none", dtype)
    special = torch.tensor([rows[1], rows[2], rows[-1]])
    others = torch.ones(m, dtype=torch.bool)
    others[special] = False
    for g, (value, _), what in zip(got, want, ("result", "saved", "saved u")):
        some = R.d(g[rows])
        assert torch.equal(torch.isnan(some), torch.isnan(value)) and torch.equal(torch.isinf(some), torch.isinf(value)), what
        assert torch.equal(some[torch.isinf(value)], value[torch.isinf(value)]), what
        assert bool(torch.isfinite(g[others.cuda()]).all()), what


@pytest.mark.parametrize("case", [c for c in FORWARD if c[1] == "f32" and c[3] in (K.TILE128, K.TILE256)], ids=K.name)
def test_ends_of_f32(gpu_lib, case):
    """The largest numbers against small ones, and numbers of 2^-100 against large ones: products of ordinary size, formed
    from three parts, or again in f32 where parts or sums are out of range."""
    import torch
    log(K.name(case))
    op, _, (m, n, k) = case[:3]
    x, ws, bs, r = operands(scaled, case, 4)
    top = torch.finfo(torch.float32).max
    x[:, 3] *= 2.0 ** 120
    x[1, 3], x[2, 3], x[3, 3] = top, -top, 2.0 ** 128 - 2.0 ** 119
    x[:, 4] *= 2.0 ** -100
    x[m // 2:, 5] *= 2.0 ** -140     # below the normal numbers: as they are
    for w in ws:
        w[:, 3] *= 2.0 ** -126
        w[:, 4] *= 2.0 ** 100
        w[:, 5] *= 2.0 ** 126
    got = run(gpu_lib, case, x, ws, bs, r, "none")
    want = R.linear(x, ws[0], bs[0], r, "none", "f32") if op == "linear" else R.gated(x, *ws, *bs, "none", "f32")
    for g, (value, bound), what in zip(got, want, ("result", "saved", "saved u")):
        beyond = value.abs() > 2 * top   # (products of both projections reach 2^252)
        value = value.masked_fill(beyond & (value > 0), float("inf")).masked_fill(beyond & (value < 0), -float("inf"))
        R.check(g, (value, bound), what)


def gradients(lib, case, t, act):
    if case[0] == "linear":
        return lib.linear_backward(t["dy"], t["x"], t["ws"][0], t["zs"][0], activation=act)
    return lib.gated_ffn_backward(t["dy"], t["x"], *t["ws"], *t["zs"], activation=act, bias=True)


def saved(make, case, seed):
    op, dtype, (m, n, k) = case[:3]
    gen, mats = generator(seed), 1 if op == "linear" else 2
    return {"x": make(gen, dtype, m, k), "dy": make(gen, dtype, m, n), "ws": [make(gen, dtype, n, k) for _ in range(mats)],
            "zs": [make(gen, dtype, m, n) for _ in range(mats)]}


NAMES = {"linear": ("dx", "dw", "db"), "gated": ("dx", "dw_gate", "dw_up", "db_gate", "db_up")}


@pytest.mark.parametrize("case", BACKWARD, ids=K.name)
def test_backward(gpu_lib, case):
    log(K.name(case))
    t = saved(normal, case, 5)
    got = gradients(gpu_lib, case, t, "gelu")
    reference = R.linear_backward if case[0] == "linear" else R.gated_backward
    for g, w, what in zip(got, reference(t["dy"], t["x"], *t["ws"], *t["zs"], "gelu", case[1]), NAMES[case[0]]):
        R.check(g, w, what)


@pytest.mark.parametrize("case", BACKWARD, ids=K.name)
def test_backward_whole_numbers(gpu_lib, case):
    import torch
    log(K.name(case))
    op, dtype, (m, n, k) = case[:3]
    t = saved(whole_numbers, case, 6)
    dy, x, zs = t["dy"].float(), t["x"].float(), [z.float() for z in t["zs"]]
    if op == "linear":
        ds = [dy * (zs[0] > 0)]
    else:
        ds = [dy * zs[1] * (zs[0] > 0), dy * zs[0].clamp(min=0)]
    want = [sum(d @ w.float() for d, w in zip(ds, t["ws"])), *(d.t() @ x for d in ds), *(d.sum(0) for d in ds)]
    want = [w.to(R.TYPES[dtype]) for w in want]
    for g, w, what in zip(gradients(gpu_lib, case, t, "relu"), want, NAMES[op]):
        assert torch.equal(g, w), what

    def inside(v):
        big = torch.full((v.shape[0] + 2, v.shape[1] + 11), float("nan"), dtype=v.dtype, device="cuda")
        view = big[1:-1, 3:3 + v.shape[1]]
        view.copy_(v)
        return view

    views = {"x": inside(t["x"]), "dy": inside(t["dy"]), "ws": [inside(w) for w in t["ws"]], "zs": [inside(z) for z in t["zs"]]}
    for g, w, what in zip(gradients(gpu_lib, case, views, "relu"), want, NAMES[op]):
        assert torch.equal(g, w), what + " of views"


@pytest.mark.parametrize("case", BACKWARD, ids=K.name)
def test_backward_not_finite(gpu_lib, case):
    """An infinite gradient reaches its row of dx, its column of the weights' gradients' rows, and nothing else."""
    import torch
    log(K.name(case))
    op, dtype, (m, n, k) = case[:3]
    t = saved(normal, case, 7)
    for v in (t["x"], *t["ws"], *t["zs"]):
        v[v == 0] = 0.5
        v.clamp_(-2, 2)
    row, column = m // 2, n - 1
    t["dy"][row, column] = float("inf")
    dx, *rest = gradients(gpu_lib, case, t, "sigmoid")
    finite = torch.isfinite(dx)
    assert not bool(finite[row].any()) and int((~finite).sum()) == k
    for v in rest:
        finite = torch.isfinite(v)
        assert not bool(finite[column].any()) and int((~finite).sum()) == v[column].numel()


@pytest.mark.parametrize("case", [c for c in BACKWARD if c[1] == "f32"], ids=K.name)
def test_backward_ends_of_f32(gpu_lib, case):
    log(K.name(case))
    t = saved(normal, case, 8)
    t["dy"][:, 0] *= 2.0 ** 100
    t["dy"][0] *= 2.0 ** -20
    for w in t["ws"]:
        w[0] *= 2.0 ** -100
    got = gradients(gpu_lib, case, t, "relu")
    reference = R.linear_backward if case[0] == "linear" else R.gated_backward
    for g, w, what in zip(got, reference(t["dy"], t["x"], *t["ws"], *t["zs"], "relu", "f32"), NAMES[case[0]]):
        R.check(g, w, what)


@pytest.mark.parametrize("case", [c for c in FORWARD if c[3] != K.ROWS], ids=K.name)
def test_equal_calls(gpu_lib, case):
    import torch
    x, ws, bs, r = operands(scaled, case, 9)
    one, two = (run(gpu_lib, case, x, ws, bs, r, "gelu") for _ in range(2))
    assert all(torch.equal(p, q) for p, q in zip(one, two))


@pytest.mark.parametrize("stride", [1 << 22, (1 << 22) + 8])   # the tiles read the first where it lies; the second is copied
@pytest.mark.parametrize("dtype,m,n,k", [("f16", 257, 4100, 40), ("bf16", 2051, 2000, 520)], ids=str)
def test_far_rows(gpu_lib, dtype, m, n, k, stride):
    """Rows of every operand and result 2^23 bytes apart or more, on tiles, forward and backward."""
    import torch
    log(f"far rows {dtype} {m} {n} {k} {stride}")
    gen = generator(10)

    def far(t):
        out = torch.empty_strided(t.shape, (stride, 1), dtype=t.dtype, device="cuda")
        return out.copy_(t)

    x, w, dy, z = (whole_numbers(gen, dtype, *s) for s in ((m, k), (n, k), (m, n), (m, n)))
    fx, fw, fdy, fz = (far(t) for t in (x, w, dy, z))
    out = far(torch.zeros_like(dy))
    gpu_lib.linear(fx, fw, None, fdy, out=out)
    assert torch.equal(out, (x.float() @ w.float().t() + dy.float()).to(x.dtype))
    gpu_lib.gated_ffn(fx, fw, fw, activation="none", out=out)
    assert torch.equal(out, (x.float() @ w.float().t()).square().to(x.dtype))
    dz = dy.float() * (z > 0)
    got = gpu_lib.linear_backward(fdy, fx, fw, fz, activation="relu")
    for g, v in zip(got, (dz @ w.float(), dz.t() @ x.float(), dz.sum(0))):
        assert torch.equal(g, v.to(x.dtype))
    dg, du = dy.float() * z.float() * (z > 0), dy.float() * z.float().clamp(min=0)
    got = gpu_lib.gated_ffn_backward(fdy, fx, fw, fw, fz, fz, activation="relu", bias=True)
    want = (dg @ w.float() + du @ w.float(), dg.t() @ x.float(), du.t() @ x.float(), dg.sum(0), du.sum(0))
    for g, v in zip(got, want):
        assert torch.equal(g, v.to(x.dtype))
