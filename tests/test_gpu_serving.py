"""The dense layers' serving forms (quantize_rows, linear_int8, moe_ffn) against 64 bits, at the sizes, types, strides and
values where they can go wrong, and whole numbers exactly."""
import pytest

import dense_reference as R
import serving_reference as S
from gpu_helpers import log

pytestmark = pytest.mark.gpu
TYPES = ["f32", "f16", "bf16"]


def generator(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(gen, dtype, *shape, std=1.0):
    import torch
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(R.TYPES[dtype])


def eights(gen, *shape):
    import torch
    return torch.randint(-128, 128, shape, generator=gen, device="cuda", dtype=torch.int8)


def some(gen, *shape, of=1.0):
    import torch
    return of * (0.5 + torch.rand(*shape, generator=gen, device="cuda"))


def inside(t, left=3, fill=None):
    """The same values as a view with rows further apart, and the tensor around it."""
    import torch
    if fill is None:
        fill = float("nan") if t.dtype.is_floating_point else 99
    big = torch.full((*t.shape[:-2], t.shape[-2] + 2, t.shape[-1] + left + 5), fill, dtype=t.dtype, device="cuda")
    view = big[..., 1:-1, left:left + t.shape[-1]]
    view.copy_(t)
    return view, big


# ---------------------------------------------------------------- quantize_rows

QUANTIZE = [(1, 1), (1, 7), (3, 16), (5, 63), (2, 64), (4, 65), (300, 128), (7, 500), (3, 1001), (9, 1664), (2, 2049), (65, 4096),
            (3, 12800), (2, 16384), (2, 16385), (2, 70001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", QUANTIZE, ids=str)
def test_quantize(gpu_lib, size, dtype):
    import torch
    log(f"quantize {size} {dtype}")
    m, k = size
    gen = generator(m * 1000 + k)
    x = normal(gen, dtype, m, k) * torch.exp(normal(gen, dtype, m, 1))
    # borders: whole numbers and a half times a scale that is a power of two
    x[m // 2] = (torch.randint(-253, 254, (k,), generator=gen, device="cuda") / 2).to(x.dtype)
    x[m // 2, k // 2] = 127.0
    want_q, want_s = S.quantize(x)
    q, s = gpu_lib.quantize_rows(x)
    assert q.dtype == torch.int8 and s.dtype == torch.float32 and q.stride(0) % 16 == 0
    assert torch.equal(R.d(s), want_s) and torch.equal(R.d(q), want_q)
    view, _ = inside(x)
    out_q, around = inside(torch.zeros_like(q), fill=77)
    out_s = torch.empty_like(s)
    got = gpu_lib.quantize_rows(view, out=(out_q, out_s))
    assert got[0] is out_q and got[1] is out_s
    assert torch.equal(R.d(out_s), want_s) and torch.equal(R.d(out_q), want_q)
    out_q.fill_(77)
    assert bool((around == 77).all()), "written outside the result"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", [5, 640, 20000])
def test_quantize_ends(gpu_lib, dtype, k):
    """Rows of zeros, of the smallest and largest numbers, with infinities and NaN."""
    import torch
    info = torch.finfo(R.TYPES[dtype])
    x = normal(generator(k), dtype, 8, k)
    x[0] = 0.0
    x[1] *= info.tiny
    x[1, 0] = info.tiny
    x[2, k - 1] = info.max
    x[3, k // 2] = float("inf")
    x[4, 0] = float("nan")
    x[5] = 0.0
    x[5, k - 1] = torch.tensor(info.tiny * (2.0 ** -10 if dtype == "f16" else 2.0 ** -7)).to(x.dtype)
    x[6] = -0.0
    q, s = gpu_lib.quantize_rows(x)
    want_q, want_s = S.quantize(x)
    assert torch.equal(torch.isnan(R.d(s)), torch.isnan(want_s))
    assert torch.equal(R.d(s).nan_to_num(7.0), want_s.nan_to_num(7.0)) and torch.equal(R.d(q), want_q)
    assert torch.isnan(s[3]) and torch.isnan(s[4]) and not q[3].any() and float(s[0]) == 2.0 ** -126


# ---------------------------------------------------------------- linear_int8

LINEAR = [(1, 1, 1), (1, 512, 1664), (2, 77, 200), (3, 8, 15), (16, 33, 64), (17, 300, 129), (19, 4096, 512), (33, 100, 1001),
          (64, 64, 16), (130, 257, 300), (256, 256, 4096), (300, 130, 5000), (777, 1365, 1001), (1024, 1024, 640), (2048, 2304, 272),
          (4100, 515, 100), (5000, 1, 300), (1, 3000, 13)]


def linear_operands(size, dtype, seed):
    m, n, k = size
    gen = generator(seed)
    return dict(q=eights(gen, m, k), xs=some(gen, m, of=0.02), w=eights(gen, n, k), ws=some(gen, n, of=0.02 * k ** -0.5),
                b=normal(gen, dtype, n), r=normal(gen, dtype, m, n))


@pytest.mark.parametrize("size", LINEAR, ids=str)
def test_linear_int8(gpu_lib, size):
    """Quantized x: every type of result, with and without each operand, and operands inside larger matrices."""
    import torch
    log(f"linear_int8 {size}")
    for at, dtype in enumerate(TYPES):
        o = linear_operands(size, dtype, at)
        act = ["gelu", "silu", "sigmoid"][at]
        want = S.linear_int8(o["q"], o["xs"], o["w"], o["ws"], o["b"], o["r"], act, dtype)
        y = gpu_lib.linear_int8(o["q"], o["w"], o["ws"], o["b"], o["r"], x_scale=o["xs"], activation=act)
        assert y.dtype == R.TYPES[dtype]
        R.check(y, want, f"{dtype} {act}")
        over = o["r"].clone()
        assert gpu_lib.linear_int8(o["q"], o["w"], o["ws"], o["b"], over, x_scale=o["xs"], activation=act, out=over) is over
        assert torch.equal(over, y), "over the residual"
        left = [3, 16, 8][at]
        out, around = inside(torch.zeros_like(y), left)
        gpu_lib.linear_int8(inside(o["q"], left)[0], inside(o["w"], left)[0], o["ws"], o["b"], inside(o["r"], left)[0],
                            x_scale=o["xs"], activation=act, out=out)
        assert torch.equal(out, y), "of views"
        out.fill_(float("nan"))
        assert bool(torch.isnan(around).all()), "written outside the result"
        plain = gpu_lib.linear_int8(o["q"], o["w"], o["ws"], x_scale=o["xs"], dtype=R.TYPES[dtype])
        R.check(plain, S.linear_int8(o["q"], o["xs"], o["w"], o["ws"], None, None, "none", dtype), f"{dtype} alone")


@pytest.mark.parametrize("size", LINEAR, ids=str)
def test_linear_int8_of_float(gpu_lib, size):
    """x quantized by the call: bit for bit what quantize_rows and the product of its results give."""
    import torch
    log(f"linear_int8 of float {size}")
    m, n, k = size
    for at, dtype in enumerate(TYPES):
        o = linear_operands(size, dtype, 10 + at)
        x = normal(generator(20 + at), dtype, m, k)
        y = gpu_lib.linear_int8(x, o["w"], o["ws"], o["b"], o["r"], activation="relu")
        q, s = gpu_lib.quantize_rows(x)
        assert torch.equal(y, gpu_lib.linear_int8(q, o["w"], o["ws"], o["b"], o["r"], x_scale=s, activation="relu"))
        R.check(y, S.linear_int8(q, s, o["w"], o["ws"], o["b"], o["r"], "relu", dtype), dtype)
        assert torch.equal(y, gpu_lib.linear_int8(inside(x)[0], inside(o["w"])[0], o["ws"], o["b"], o["r"], activation="relu"))


@pytest.mark.parametrize("size", [(1, 70, 131071), (40, 300, 131071), (600, 600, 131071)], ids=str)
def test_linear_int8_longest_sums(gpu_lib, size):
    """The largest sum that 32 bits hold: k of 131071 and all values -128."""
    import torch
    m, n, k = size
    q = torch.full((m, k), -128, dtype=torch.int8, device="cuda")
    w = torch.full((n, k), -128, dtype=torch.int8, device="cuda")
    q[0], w[1] = 127, 127
    one = torch.ones(max(m, n), device="cuda")
    y = gpu_lib.linear_int8(q, w, one[:n], x_scale=one[:m], dtype=torch.float32)
    a, b = q[:, 0].double(), w[:, 0].double()
    assert torch.equal(y, (k * a[:, None] * b).float())


def test_linear_int8_rows_that_are_not_finite(gpu_lib):
    """A row of x with NaN or an infinity gives NaN there and nowhere else; so does a scale that is NaN."""
    import torch
    gen = generator(5)
    for m, n, k in ((5, 40, 100), (700, 300, 512)):
        x, w, ws = normal(gen, "bf16", m, k), eights(gen, n, k), some(gen, n)
        x[1, 3], x[m - 1, k - 1] = float("inf"), float("nan")
        y = gpu_lib.linear_int8(x, w, ws, activation="relu")
        bad = torch.zeros(m, dtype=torch.bool, device="cuda")
        bad[1] = bad[m - 1] = True
        assert bool(torch.isnan(y[bad]).all()) and bool(torch.isfinite(y[~bad]).all())
        ws[n - 1] = float("nan")
        y = gpu_lib.linear_int8(x, w, ws)
        assert bool(torch.isnan(y[:, n - 1]).all()) and bool(torch.isfinite(y[~bad][:, :n - 1]).all())


# ---------------------------------------------------------------- moe_ffn

# rows, f, d, experts, top_k
MOE = [(1, 1, 1, 1, 1), (1, 16, 16, 2, 1), (1, 40, 24, 4, 2), (1, 704, 256, 16, 4), (2, 333, 1001, 7, 3), (4, 128, 320, 8, 8),
       (5, 64, 130, 3, 2), (17, 48, 200, 5, 5), (19, 100, 64, 8, 2), (33, 65, 33, 40, 1), (64, 256, 128, 32, 4), (70, 31, 96, 2, 2),
       (200, 33, 65, 16, 4), (7, 24, 40, 130, 32), (300, 40, 48, 6, 3), (600, 32, 64, 3, 2), (1, 2000, 72, 2, 2), (9, 8, 4100, 1024, 8),
       (20, 700, 96, 4, 2), (70, 500, 100, 3, 2), (12, 1500, 300, 2, 1), (2, 400, 2100, 4, 2), (130, 72, 60, 2, 2), (40, 6000, 17, 8, 2),
       (2, 300, 9000, 6, 2)]


def moe_operands(size, dtype, seed, eight):
    m, f, dim, e, _ = size
    gen = generator(seed)
    o = dict(x=normal(gen, dtype, m, dim), router=normal(gen, dtype, e, dim, std=2.0 * dim ** -0.5))
    if eight:
        o["ws"] = [eights(gen, e, f, dim), eights(gen, e, f, dim), eights(gen, e, dim, f)]
        o["scales"] = tuple(some(gen, *w.shape[:2], of=0.02 * w.shape[2] ** -0.5) for w in o["ws"])
    else:
        o["ws"] = [normal(gen, dtype, e, r, c, std=c ** -0.5) for r, c in ((f, dim), (f, dim), (dim, f))]
        o["scales"] = None
    return o


@pytest.mark.parametrize("eight", [False, True], ids=["float", "int8"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", MOE, ids=str)
def test_moe(gpu_lib, size, dtype, eight):
    import torch
    log(f"moe {size} {dtype} {eight}")
    top = size[4]
    o = moe_operands(size, dtype, 1, eight)
    act = {"f32": "gelu", "f16": "silu", "bf16": "silu"}[dtype]
    y, chosen, share = gpu_lib.moe_ffn(o["x"], o["router"], *o["ws"], top_k=top, scales=o["scales"], activation=act, routing=True)
    want, experts, shares = S.moe(o["x"], o["router"], *o["ws"], top, act, dtype, o["scales"])
    assert chosen.dtype == torch.int32 and torch.equal(chosen.cpu(), experts)
    R.check(share, shares, "shares")
    R.check(y, want, "result")
    # without the routing, from views, into a view
    out, around = inside(torch.zeros_like(y))
    ws = [inside(w)[0] for w in o["ws"]]
    assert gpu_lib.moe_ffn(inside(o["x"])[0], inside(o["router"])[0], *ws, top_k=top, scales=o["scales"], activation=act,
                           out=out) is out
    assert torch.equal(out, y), "of views"
    out.fill_(float("nan"))
    assert bool(torch.isnan(around).all()), "written outside the result"


@pytest.mark.parametrize("eight", [False, True], ids=["float", "int8"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(1, 40, 600, 256, 8), (2, 33, 65, 64, 6), (3, 24, 1500, 17, 17), (12, 130, 48, 20, 2), (15, 16, 33, 17, 1),
                                  (1, 20, 7, 1024, 32), (256, 17, 20, 18, 3), (257, 17, 20, 18, 3)], ids=str)
def test_moe_many_experts(gpu_lib, size, dtype, eight):
    """Logits in a launch of their own, and their experts picked in the next one's workgroups or in a launch too."""
    test_moe(gpu_lib, size, dtype, eight)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(65, 500, 1100, 4, 2), (70, 501, 1101, 4, 1), (800, 300, 1000, 8, 4), (700, 100, 700, 64, 2),
                                  (100, 64, 1100, 32, 16), (1300, 20, 3000, 40, 1), (90, 4000, 33, 17, 3), (66, 31, 3001, 24, 24)], ids=str)
def test_moe_by_experts(gpu_lib, size, dtype):
    """Down projections by experts: more than 64 rows and 4 MB of weights; uses in one list and several, tiles full and not."""
    test_moe(gpu_lib, size, dtype, False)


@pytest.mark.parametrize("dtype", TYPES)
def test_moe_shares_over_all(gpu_lib, dtype):
    size = (21, 40, 72, 9, 3)
    o = moe_operands(size, dtype, 2, False)
    y, chosen, share = gpu_lib.moe_ffn(o["x"], o["router"], *o["ws"], top_k=3, renormalize=False, routing=True)
    want, experts, shares = S.moe(o["x"], o["router"], *o["ws"], 3, "silu", dtype, renormalize=False)
    assert (chosen.cpu() == experts).all() and float(share.sum(1).max()) < 1.0
    R.check(share, shares, "shares")
    R.check(y, want, "result")


def test_moe_ties_and_values_that_are_not_finite(gpu_lib):
    """Ties go to the lowest expert; NaN among a row's logits makes that row NaN and no other; -inf is never taken."""
    import torch
    for m in (4, 40):
        o = moe_operands((m, 24, 32, 6, 2), "f32", 3, False)
        o["router"][4] = o["router"][1]
        o["router"][5] = o["router"][1]
        y, chosen, _ = gpu_lib.moe_ffn(o["x"], o["router"], *o["ws"], top_k=4, routing=True)
        want, experts, _ = S.moe(o["x"], o["router"], *o["ws"], 4, "silu", "f32")
        assert torch.equal(chosen.cpu(), experts)
        R.check(y, want, "ties")
        zero = torch.zeros_like(o["router"])
        _, chosen, share = gpu_lib.moe_ffn(o["x"], zero, *o["ws"], top_k=3, routing=True)
        assert torch.equal(chosen.cpu(), torch.tensor([[0, 1, 2]] * m, dtype=torch.int32))
        assert bool(((share - 1 / 3).abs() < 1e-7).all())
        o["x"][2, 5] = float("nan")
        o["x"][3, 0] = float("inf")
        y, chosen, share = gpu_lib.moe_ffn(o["x"], o["router"], *o["ws"], top_k=2, routing=True)
        bad = torch.zeros(m, dtype=torch.bool, device="cuda")
        bad[2] = bad[3] = True
        assert bool(torch.isnan(y[bad]).all()) and bool(torch.isfinite(y[~bad]).all())
        assert chosen[2].tolist() == [0, 1] and bool(torch.isnan(share[2]).all())
        assert bool(((chosen >= 0) & (chosen < 6)).all())


def test_moe_a_row_alone(gpu_lib):
    """A row's result comes from that row and its experts, also beside a row of NaN; equal calls give equal bits."""
    import torch
    for dtype in TYPES:
        o = moe_operands((30, 70, 90, 4, 2), dtype, 4, False)
        o["x"][5] = float("nan")
        y = gpu_lib.moe_ffn(o["x"], o["router"], *o["ws"], top_k=2)
        again = gpu_lib.moe_ffn(o["x"], o["router"], *o["ws"], top_k=2)
        rows = [i for i in range(30) if i != 5]
        assert torch.equal(y[rows], again[rows]), "equal calls, equal bits"
        want, _, _ = S.moe(o["x"][rows], o["router"], *o["ws"], 2, "silu", dtype)
        R.check(y[rows], want, "beside NaN")


def test_moe_experts_not_taken_are_not_used(gpu_lib):
    import torch
    o = moe_operands((6, 40, 48, 8, 2), "bf16", 6, False)
    y, chosen, _ = gpu_lib.moe_ffn(o["x"], o["router"], *o["ws"], top_k=2, routing=True)
    free = [e for e in range(8) if e not in set(chosen.flatten().tolist())]
    for e in free:
        for w in o["ws"]:
            w[e] = float("nan")
    assert torch.equal(y, gpu_lib.moe_ffn(o["x"], o["router"], *o["ws"], top_k=2))


def test_no_rows(gpu_lib):
    import torch
    o = moe_operands((1, 40, 48, 8, 2), "f16", 6, False)
    y, chosen, share = gpu_lib.moe_ffn(o["x"][:0], o["router"], *o["ws"], top_k=2, routing=True)
    assert y.shape == (0, 48) and chosen.shape == (0, 2) and share.shape == (0, 2)
    q, s = gpu_lib.quantize_rows(o["x"][:0])
    assert q.shape == (0, 48) and s.shape == (0,)
    w, ws = gpu_lib.quantize_rows(o["router"])
    assert gpu_lib.linear_int8(o["x"][:0], w, ws).shape == (0, 8)
    assert gpu_lib.linear_int8(q, w, ws, x_scale=s).dtype == torch.bfloat16


# ---------------------------------------------------------------- together

def layers(lib, p, x):
    """As a server calls them: 8-bit layer, experts of 8 bits with a skip connection, 8-bit head."""
    y = lib.linear_int8(x, *p["first"], p["bias"], activation="relu")
    z = lib.moe_ffn(y, p["router"], *p["ws"], top_k=2, scales=p["scales"])
    z += y
    return lib.linear_int8(z, *p["last"], activation="sigmoid")


def weights(lib, dtype, gen, k=200, d=96, f=160, e=6):
    p = {"first": lib.quantize_rows(normal(gen, dtype, d, k, std=k ** -0.5)), "bias": normal(gen, dtype, d),
         "router": normal(gen, dtype, e, d, std=2 * d ** -0.5), "last": lib.quantize_rows(normal(gen, dtype, 1, d, std=d ** -0.5))}
    made = [lib.quantize_rows(normal(gen, dtype, e * r, c, std=c ** -0.5)) for r, c in ((f, d), (f, d), (d, f))]
    p["ws"] = [q.unflatten(0, (e, -1)) for q, _ in made]
    p["scales"] = tuple(s.view(e, -1) for _, s in made)
    return p


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 23, 300])
def test_together(gpu_lib, m, dtype):
    """Each step within its bound of 64 bits on the inputs that it was given."""
    gen = generator(m)
    p = weights(gpu_lib, dtype, gen)
    x = normal(gen, dtype, m, 200)
    y = gpu_lib.linear_int8(x, *p["first"], p["bias"], activation="relu")
    R.check(y, S.linear_int8(*S.quantize(x), *p["first"], p["bias"], None, "relu", dtype), "first")
    z, chosen, _ = gpu_lib.moe_ffn(y, p["router"], *p["ws"], top_k=2, scales=p["scales"], routing=True)
    want, experts, _ = S.moe(y, p["router"], *p["ws"], 2, "silu", dtype, p["scales"])
    assert (chosen.cpu() == experts).all()
    R.check(z, want, "experts")
    z += y
    last = gpu_lib.linear_int8(z, *p["last"], activation="sigmoid")
    R.check(last, S.linear_int8(*S.quantize(z), *p["last"], None, None, "sigmoid", dtype), "last")


def test_captured_and_replayed(gpu_lib):
    """The whole run as a graph, replayed with other inputs, with eager work between."""
    import torch
    gen = generator(9)
    p = weights(gpu_lib, "bf16", gen)
    for m in (1, 40, 300):
        x = normal(gen, "bf16", m, 200)
        layers(gpu_lib, p, x)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = layers(gpu_lib, p, x)
        for _ in range(4):
            x.copy_(normal(gen, "bf16", m, 200))
            eager = layers(gpu_lib, p, x)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, eager)


def test_streams(gpu_lib):
    """Calls on two streams at once, each with the results that it has alone."""
    import torch
    gen = generator(10)
    p = weights(gpu_lib, "f16", gen)
    xs = [normal(gen, "f16", m, 200) for m in (3, 150)]
    alone = [layers(gpu_lib, p, x) for x in xs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for at, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[at].append(layers(gpu_lib, p, xs[at]))
    q, scale = gpu_lib.quantize_rows(xs[1], stream=streams[0])
    y = gpu_lib.linear_int8(q, *p["first"], p["bias"], x_scale=scale, stream=streams[0])
    z = gpu_lib.moe_ffn(y, p["router"], *p["ws"], top_k=2, scales=p["scales"], stream=streams[0].cuda_stream)
    torch.cuda.synchronize()
    for want, many in zip(alone, got):
        assert all(torch.equal(want, g) for g in many)
    y2 = gpu_lib.linear_int8(xs[1], *p["first"], p["bias"])
    assert torch.equal(y, y2)
    assert torch.equal(z, gpu_lib.moe_ffn(y2, p["router"], *p["ws"], top_k=2, scales=p["scales"]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", [1, 3, 4, 5, 12, 13, 31, 100])
def test_rows_that_end_inside_16_bytes(gpu_lib, dtype, k):
    """Rows that start at multiples of 16 bytes and end inside of some: what lies behind them, NaN, is not used."""
    import torch
    gen = generator(k)
    m, e = 5, 4

    def padded(t):
        big = torch.full((*t.shape[:-1], (t.shape[-1] + 15) // 16 * 16), float("nan") if t.is_floating_point() else 77, dtype=t.dtype, device="cuda")
        big[..., :t.shape[-1]] = t
        return big[..., :t.shape[-1]]

    x, w, ws = padded(normal(gen, dtype, m, k)), padded(eights(gen, 40, k)), some(gen, 40)
    q, s = gpu_lib.quantize_rows(x)
    want_q, want_s = S.quantize(x)
    assert torch.equal(R.d(q), want_q) and torch.equal(R.d(s), want_s)
    R.check(gpu_lib.linear_int8(x, w, ws), S.linear_int8(q, s, w, ws, None, None, "none", dtype), "quantized inside")
    many = padded(normal(gen, dtype, 300, k))
    R.check(gpu_lib.linear_int8(many, w, ws), S.linear_int8(*S.quantize(many), w, ws, None, None, "none", dtype), "quantized before")
    for f in (7, 40):
        router = padded(normal(gen, dtype, e, k))
        mats = [padded(normal(gen, dtype, e, f, k)), padded(normal(gen, dtype, e, f, k)), padded(normal(gen, dtype, e, k, f))]
        for rows in (x, many[:70]):
            want, _, _ = S.moe(rows, router, *mats, 2, "silu", dtype)
            R.check(gpu_lib.moe_ffn(rows, router, *mats, top_k=2), want, "experts")
        eight = [padded(eights(gen, *t.shape)) for t in mats]
        scales = tuple(some(gen, *t.shape[:2], of=0.01) for t in mats)
        want, _, _ = S.moe(x, router, *eight, 2, "silu", dtype, scales)
        R.check(gpu_lib.moe_ffn(x, router, *eight, top_k=2, scales=scales), want, "experts of 8 bits")
