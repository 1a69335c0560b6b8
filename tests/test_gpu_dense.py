"""The dense layers on the GPU against their formulas in 64 bits (dense_reference.py): every type, activation and
direction, sizes from one row to several tiles with odd remainders, strides, what lies beside the operands in memory,
streams, graphs and repeatability."""
import pytest

import dense_reference as R
from gpu_helpers import log

pytestmark = pytest.mark.gpu

DTYPES = ["f32", "f16", "bf16"]
ACTS = ["none", "relu", "sigmoid", "silu", "gelu"]
# one element, one row, tails of every tile size on each axis, whole tiles, few rows of a wide layer, one column
SIZES = [(1, 1, 1), (1, 512, 1664), (2, 3, 5), (7, 65, 31), (16, 64, 64), (17, 100, 13), (19, 352, 1024), (33, 130, 257),
         (64, 1, 256), (65, 7, 129), (128, 128, 128), (129, 257, 65), (256, 256, 320), (300, 1, 77), (301, 515, 264),
         (513, 13, 1000), (1030, 260, 40), (77, 1000, 2056)]


def make(dtype, seed, *shapes):
    """Device tensors of normal values, of std 1 / sqrt(columns) or so: products of order one."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    out = []
    for shape, std in shapes:
        out.append(None if shape is None else (torch.randn(shape, generator=gen, dtype=torch.float32) * std).to(R.TYPES[dtype]).cuda())
    return out


def layer(dtype, seed, m, n, k, bias=True, residual=False):
    return make(dtype, seed, ((m, k), 1.0), ((n, k), k ** -0.5), ((n,) if bias else None, 0.3),
                ((m, n) if residual else None, 1.0))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_linear_sizes(gpu_lib, size, dtype):
    m, n, k = size
    log(f"linear {size} {dtype}")
    x, w, b, r = layer(dtype, 1, m, n, k, residual=True)
    y, z = gpu_lib.linear(x, w, b, r, activation="silu", save=True)
    want_y, want_z = R.linear(x, w, b, r, "silu", dtype)
    R.check(z, want_z, "z")
    R.check(y, want_y, "y")
    plain = gpu_lib.linear(x, w)
    R.check(plain, R.linear(x, w, None, None, "none", dtype)[0], "x W^T")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("bias,residual,save", [(False, False, False), (True, False, True), (False, True, False), (True, True, True)])
def test_linear_epilogues(gpu_lib, act, dtype, bias, residual, save):
    for m, n, k in [(5, 48, 72), (150, 136, 96)]:
        log(f"linear {act} {dtype} bias {bias} residual {residual} save {save} rows {m}")
        x, w, b, r = layer(dtype, 2, m, n, k, bias, residual)
        out = gpu_lib.linear(x, w, b, r, activation=act, save=save)
        want_y, want_z = R.linear(x, w, b, r, act, dtype)
        if save:
            R.check(out[1], want_z, "z")
        R.check(out[0] if save else out, want_y, "y")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_linear_backward_sizes(gpu_lib, size, dtype):
    m, n, k = size
    log(f"linear_backward {size} {dtype}")
    x, w, dy, z = make(dtype, 3, ((m, k), 1.0), ((n, k), k ** -0.5), ((m, n), 0.5), ((m, n), 1.0))
    got = gpu_lib.linear_backward(dy, x, w, z, activation="gelu")
    for g, want, what in zip(got, R.linear_backward(dy, x, w, z, "gelu", dtype), ("dx", "dw", "db")):
        R.check(g, want, what)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ACTS)
def test_linear_backward_activations(gpu_lib, act, dtype):
    m, n, k = 200, 72, 120
    log(f"linear_backward {act} {dtype}")
    x, w, dy, z = make(dtype, 4, ((m, k), 1.0), ((n, k), k ** -0.5), ((m, n), 0.5), ((m, n), 1.5))
    z[::7, ::3] = 0.0
    z[3, :8] = 30.0
    z[4, :8] = -30.0
    want = R.linear_backward(dy, x, w, z, act, dtype)
    for dx, dw, db in [(1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)]:
        got = gpu_lib.linear_backward(dy, x, w, z if act != "none" else None, activation=act, bias=bool(db),
                                      need_dx=bool(dx), need_dw=bool(dw))
        for g, v, yes, what in zip(got, want, (dx, dw, db), ("dx", "dw", "db")):
            assert (g is not None) == bool(yes)
            if yes:
                R.check(g, v, what)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gated_sizes(gpu_lib, size, dtype):
    m, n, k = size
    log(f"gated_ffn {size} {dtype}")
    x, wg, wu, bg, bu = make(dtype, 5, ((m, k), 1.0), ((n, k), k ** -0.5), ((n, k), k ** -0.5), ((n,), 0.3), ((n,), 0.3))
    got = gpu_lib.gated_ffn(x, wg, wu, bg, bu, save=True)
    for g, want, what in zip(got, R.gated(x, wg, wu, bg, bu, "silu", dtype), "hgu"):
        R.check(g, want, what)
    R.check(gpu_lib.gated_ffn(x, wg, wu), R.gated(x, wg, wu, None, None, "silu", dtype)[0], "h without biases")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ACTS)
def test_gated_activations(gpu_lib, act, dtype):
    for m, n, k in [(9, 40, 200), (140, 200, 104)]:
        log(f"gated_ffn {act} {dtype} rows {m}")
        x, wg, wu, bg, bu = make(dtype, 6, ((m, k), 1.0), ((n, k), k ** -0.5), ((n, k), k ** -0.5), ((n,), 0.3), ((n,), 0.3))
        for b0, b1 in [(bg, bu), (bg, None), (None, bu)]:
            R.check(gpu_lib.gated_ffn(x, wg, wu, b0, b1, activation=act), R.gated(x, wg, wu, b0, b1, act, dtype)[0], "h")
        dh, g, u = make(dtype, 7, ((m, n), 0.5), ((m, n), 1.5), ((m, n), 1.0))
        got = gpu_lib.gated_ffn_backward(dh, x, wg, wu, g, u, activation=act, bias=True)
        for v, want, what in zip(got, R.gated_backward(dh, x, wg, wu, g, u, act, dtype), ("dx", "dwg", "dwu", "dbg", "dbu")):
            R.check(v, want, what)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_gated_backward_sizes(gpu_lib, size, dtype):
    m, n, k = size
    log(f"gated_ffn_backward {size} {dtype}")
    x, wg, wu, dh, g, u = make(dtype, 8, ((m, k), 1.0), ((n, k), k ** -0.5), ((n, k), k ** -0.5), ((m, n), 0.5),
                               ((m, n), 1.0), ((m, n), 1.0))
    want = R.gated_backward(dh, x, wg, wu, g, u, "silu", dtype)
    names = ("dx", "dwg", "dwu", "dbg", "dbu")
    for v, wv, what in zip(gpu_lib.gated_ffn_backward(dh, x, wg, wu, g, u, bias=True), want, names):
        R.check(v, wv, what)
    got = gpu_lib.gated_ffn_backward(dh, x, wg, wu, g, u, need_dx=False)
    assert got[0] is None and got[3] is None and got[4] is None
    R.check(got[1], want[1], "dwg alone")
    R.check(got[2], want[2], "dwu alone")
    got = gpu_lib.gated_ffn_backward(dh, x, wg, wu, g, u, need_dw=False)
    assert got[1] is None
    R.check(got[0], want[0], "dx alone")


def _inside(t, left, right, top=1, bottom=1, poison=float("nan")):
    """t as a view into a larger matrix whose other elements are poison."""
    import torch
    big = torch.full((t.shape[0] + top + bottom, t.shape[1] + left + right), poison, dtype=t.dtype, device=t.device)
    view = big[top:top + t.shape[0], left:left + t.shape[1]]
    view.copy_(t)
    return view, big


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("left,right", [(8, 8), (1, 0), (3, 2), (4, 12)])
@pytest.mark.parametrize("size", [(6, 40, 72), (140, 136, 200), (67, 53, 101)], ids=str)
def test_views_of_larger_matrices(gpu_lib, size, dtype, left, right):
    """Rows of any stride and alignment; NaN all around the operands reaches no result, and nothing is written
    outside the results."""
    import torch
    m, n, k = size
    log(f"views {size} {dtype} margins {left} {right}")
    x, w, wu, b, r, dy, z, u = make(dtype, 9, ((m, k), 1.0), ((n, k), k ** -0.5), ((n, k), k ** -0.5), ((n,), 0.3), ((m, n), 1.0),
                                    ((m, n), 0.5), ((m, n), 1.0), ((m, n), 1.0))
    vx, vw, vwu, vr, vdy, vz, vu = (_inside(t, left, right)[0] for t in (x, w, wu, r, dy, z, u))
    vb = torch.full((n + left + right,), float("nan"), dtype=b.dtype, device="cuda")[left:left + n]
    vb.copy_(b)
    out, around = _inside(torch.zeros_like(r), left, right, poison=7.0)
    gpu_lib.linear(vx, vw, vb, vr, activation="gelu", out=out)
    R.check(out, R.linear(x, w, b, r, "gelu", dtype)[0], "y")
    mask = torch.ones_like(around, dtype=torch.bool)
    mask[1:1 + m, left:left + n] = False
    assert bool((around[mask] == 7.0).all()), "written outside the result"
    gpu_lib.gated_ffn(vx, vw, vwu, vb, None, out=out)
    R.check(out, R.gated(x, w, wu, b, None, "silu", dtype)[0], "h")
    assert bool((around[mask] == 7.0).all()), "written outside the result"
    for v, want in zip(gpu_lib.linear_backward(vdy, vx, vw, vz, activation="silu"), R.linear_backward(dy, x, w, z, "silu", dtype)):
        R.check(v, want, "linear_backward")
    for v, want in zip(gpu_lib.linear_backward(vdy, vx, vw), R.linear_backward(dy, x, w, None, "none", dtype)):
        R.check(v, want, "linear_backward without activation")
    for v, want in zip(gpu_lib.gated_ffn_backward(vdy, vx, vw, vwu, vz, vu, bias=True),
                       R.gated_backward(dy, x, w, wu, z, u, "silu", dtype)):
        R.check(v, want, "gated_ffn_backward")


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinities_and_nan_stay_where_they_belong(gpu_lib, dtype):
    """An infinity or NaN in a row of x reaches that row's results only, as the sum of products in 64 bits has it;
    likewise a row of weights its column, in every size class."""
    import torch
    for m, n, k in [(3, 64, 64), (150, 264, 200)]:
        log(f"not finite {dtype} rows {m}")
        x, w, dy = make(dtype, 10, ((m, k), 1.0), ((n, k), k ** -0.5), ((m, n), 0.5))
        w[w == 0] = 0.5
        x[x == 0] = 0.5
        x[1, 5] = float("inf")
        x[2, k - 1] = float("nan")
        w[7, 3] = float("-inf")
        # whole powers of two among the finite factors: nothing is left of them but their leading bit
        w[:, 5] = 1.0
        x[:, 3] = 2.0
        want = R.linear(x, w, None, None, "none", dtype)[0]
        got = gpu_lib.linear(x, w)
        v = want[0]
        assert torch.equal(torch.isnan(R.d(got)), torch.isnan(v))
        assert torch.equal(torch.isinf(R.d(got)), torch.isinf(v))
        assert torch.equal(R.d(got)[torch.isinf(v)], v[torch.isinf(v)])
        fine = torch.isfinite(v)
        keep = [i for i in range(m) if i not in (1, 2)]
        R.check(got[keep][:, :7], R.linear(x[keep], w[:7], None, None, "none", dtype)[0], "rows beside them")
        assert bool(fine[keep][:, :7].all())
        dx, dw, _ = gpu_lib.linear_backward(dy, x, w)
        vdx, vdw = R.d(dy) @ R.d(w), R.d(dy).t() @ R.d(x)
        assert torch.equal(torch.isnan(R.d(dx)), torch.isnan(vdx)) and torch.equal(torch.isinf(R.d(dx)), torch.isinf(vdx))
        assert torch.equal(torch.isnan(R.d(dw)), torch.isnan(vdw)) and torch.equal(torch.isinf(R.d(dw)), torch.isinf(vdw))


@pytest.mark.parametrize("dtype", DTYPES)
def test_integers_are_exact(gpu_lib, dtype):
    """Small whole numbers: every product and sum is exact in 32 bits, so results are equal, not near."""
    import torch
    gen = torch.Generator().manual_seed(11)
    for m, n, k in [(5, 72, 200), (140, 264, 128), (515, 40, 88)]:
        log(f"integers {dtype} {m} {n} {k}")
        x, w, dy = (torch.randint(-2, 3, s, generator=gen).to(R.TYPES[dtype]).cuda() for s in ((m, k), (n, k), (m, n)))
        assert torch.equal(gpu_lib.linear(x, w).cpu(), (R.d(x) @ R.d(w).t()).to(R.TYPES[dtype]))
        dx, dw, db = gpu_lib.linear_backward(dy, x, w)
        assert torch.equal(dx.cpu(), (R.d(dy) @ R.d(w)).to(R.TYPES[dtype]))
        assert torch.equal(dw.cpu(), (R.d(dy).t() @ R.d(x)).to(R.TYPES[dtype]))
        assert torch.equal(db.cpu(), R.d(dy).sum(0).to(R.TYPES[dtype]))
        h, g, u = gpu_lib.gated_ffn(x, w, w.flip(0).contiguous(), activation="relu", save=True)
        g64 = R.d(x) @ R.d(w).t()
        assert torch.equal(g.cpu(), g64.to(R.TYPES[dtype])) and torch.equal(u.cpu(), g64.flip(1).to(R.TYPES[dtype]))


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_rows(gpu_lib, dtype):
    import torch
    log(f"no rows {dtype}")
    x, w, b, dy = make(dtype, 12, ((0, 24), 1.0), ((40, 24), 1.0), ((40,), 1.0), ((0, 40), 1.0))
    assert gpu_lib.linear(x, w, b, activation="relu").shape == (0, 40)
    assert [t.shape[0] for t in gpu_lib.gated_ffn(x, w, w, save=True)] == [0, 0, 0]
    dx, dw, db = gpu_lib.linear_backward(dy, x, w, dy, activation="relu")
    assert dx.shape == (0, 24) and bool((dw == 0).all()) and bool((db == 0).all())
    dx, dwg, dwu, dbg, dbu = gpu_lib.gated_ffn_backward(dy, x, w, w, dy, dy, bias=True)
    assert dx.shape == (0, 24) and all(bool((t == 0).all()) for t in (dwg, dwu, dbg, dbu))
    torch.cuda.synchronize()


def test_long_reductions(gpu_lib):
    """Sums over many rows or columns with few results: split over the GPU and joined."""
    for dtype, m, n, k in [("bf16", 20000, 24, 40), ("f32", 9001, 7, 13), ("f16", 8, 16, 12800), ("f32", 3, 5, 9000), ("bf16", 40, 9000, 24)]:
        log(f"long {dtype} {m} {n} {k}")
        x, w, b, dy = make(dtype, 13, ((m, k), 1.0), ((n, k), k ** -0.5), ((n,), 0.3), ((m, n), 0.1))
        y, z = gpu_lib.linear(x, w, b, activation="gelu", save=True)
        want = R.linear(x, w, b, None, "gelu", dtype)
        R.check(y, want[0], "y")
        R.check(z, want[1], "z")
        for v, wv in zip(gpu_lib.linear_backward(dy, x, w), R.linear_backward(dy, x, w, None, "none", dtype)):
            R.check(v, wv, "linear_backward")
        R.check(gpu_lib.gated_ffn(x, w, w, b), R.gated(x, w, w, b, None, "silu", dtype)[0], "h")


def test_offsets_beyond_32_bits(gpu_lib):
    """Rows 2^21 elements apart: the last ones lie beyond 2^31 elements, thus beyond 2^32 bytes."""
    import torch
    log("offsets beyond 32 bits")
    m, n, k, ld = 1100, 48, 64, 1 << 21
    x, w, b, dy = make("bf16", 14, ((m, k), 1.0), ((n, k), 0.125), ((n,), 0.3), ((m, n), 0.5))
    far = torch.empty_strided((m, k), (ld, 1), dtype=torch.bfloat16, device="cuda")
    far.copy_(x)
    out = torch.empty_strided((m, n), (ld, 1), dtype=torch.bfloat16, device="cuda")
    gpu_lib.linear(far, w, b, out=out)
    R.check(out, R.linear(x, w, b, None, "none", "bf16")[0], "y")
    fdy = torch.empty_strided((m, n), (ld, 1), dtype=torch.bfloat16, device="cuda")
    fdy.copy_(dy)
    for v, want in zip(gpu_lib.linear_backward(fdy, far, w), R.linear_backward(dy, x, w, None, "none", "bf16")):
        R.check(v, want, "linear_backward")


def test_residual_in_place(gpu_lib):
    log("y written over the residual")
    for m in (4, 200):
        x, w, b, r = layer("bf16", 15, m, 96, 64, residual=True)
        want = R.linear(x, w, b, r, "silu", "bf16")[0]
        assert gpu_lib.linear(x, w, b, r, activation="silu", out=r) is r
        R.check(r, want, "y")


@pytest.mark.parametrize("dtype", DTYPES)
def test_equal_calls_give_equal_bits(gpu_lib, dtype):
    import torch
    log(f"repeatability {dtype}")
    for m, n, k in [(1, 64, 4096), (3000, 40, 72), (260, 300, 520)]:
        x, w, b, dy, z = make(dtype, 16, ((m, k), 1.0), ((n, k), k ** -0.5), ((n,), 0.3), ((m, n), 0.5), ((m, n), 1.0))
        one = (gpu_lib.linear(x, w, b, activation="gelu"), *gpu_lib.linear_backward(dy, x, w, z, activation="gelu"),
               *gpu_lib.gated_ffn_backward(dy, x, w, w, z, dy, bias=True))
        two = (gpu_lib.linear(x, w, b, activation="gelu"), *gpu_lib.linear_backward(dy, x, w, z, activation="gelu"),
               *gpu_lib.gated_ffn_backward(dy, x, w, w, z, dy, bias=True))
        assert all(torch.equal(p, q) for p, q in zip(one, two))


def test_streams(gpu_lib):
    """Calls on side streams, given as an object, as a raw handle or as the current one, at once."""
    import torch
    log("streams")
    x, w, b, dy, z = make("f16", 17, ((700, 128), 1.0), ((96, 128), 0.1), ((96,), 0.3), ((700, 96), 0.5), ((700, 96), 1.0))
    want = [R.linear(x, w, b, None, "silu", "f16")[0], *R.linear_backward(dy, x, w, z, "silu", "f16")]
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(5):
        for s, arg in zip(streams, (streams[0], streams[1].cuda_stream, None)):
            with torch.cuda.stream(s) if arg is None else torch.cuda.stream(torch.cuda.current_stream()):
                got.append((gpu_lib.linear(x, w, b, activation="silu", stream=arg),
                            *gpu_lib.linear_backward(dy, x, w, z, activation="silu", stream=arg)))
    torch.cuda.synchronize()
    for result in got:
        for v, wv in zip(result, want):
            R.check(v, wv, "side stream")


def test_graph_replays_match_eager(gpu_lib):
    """Every call captured in one graph; replayed over other inputs with eager work between the replays."""
    import torch
    log("graph")
    m, n, k = 530, 72, 200

    def inputs(seed):
        return make("bf16", seed, ((m, k), 1.0), ((n, k), k ** -0.5), ((n,), 0.3), ((m, n), 0.5), ((m, n), 1.0), ((m, n), 1.0))

    def calls(x, w, b, dy, z, u):
        return (gpu_lib.linear(x, w, b, dy, activation="gelu"), *gpu_lib.linear_backward(dy, x, w, z, activation="gelu"),
                *gpu_lib.gated_ffn(x, w, w, b, save=True), *gpu_lib.gated_ffn_backward(dy, x, w, w, z, u, bias=True),
                gpu_lib.linear(x[:3], w, b), gpu_lib.gated_ffn(x[:3], w, w))

    held = inputs(20)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(*held)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls(*held)
    for rep in range(4):
        fresh = inputs(30 + rep)
        for h, f in zip(held, fresh):
            h.copy_(f)
        graph.replay()
        torch.cuda.synchronize()
        eager = calls(*fresh)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, eager)), f"replay {rep} differs"


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(gpu_lib, act):
    """The gradients of L = sum(c * y) in f32, from sums the forward calls saved, against central differences of L in
    64 bits.  With step h the differences are off by h^2 / 6 times the third derivative (of order one) and 1e-16 / h."""
    import torch
    log(f"differences {act}")
    m, n, k, h = 5, 6, 7, 1e-5
    x, w, wu, b, bu, c = make("f32", 18, ((m, k), 1.0), ((n, k), 0.4), ((n, k), 0.4), ((n,), 0.3), ((n,), 0.3), ((m, n), 1.0))
    y, z = gpu_lib.linear(x, w, b, activation=act, save=True)
    got = gpu_lib.linear_backward(c, x, w, z, activation=act)
    _, g, u = gpu_lib.gated_ffn(x, w, wu, b, bu, activation=act, save=True)
    got_gated = gpu_lib.gated_ffn_backward(c, x, w, wu, g, u, activation=act, bias=True)
    X, W, WU, B, BU, C = (R.d(t) for t in (x, w, wu, b, bu, c))
    if act == "relu":   # not differentiable at 0: no sum within the step of it
        assert float((X @ W.t() + B).abs().min()) > 1e-3

    def loss(X, W, B):
        return (C * R.act(X @ W.t() + B, act)).sum()

    def gated_loss(X, W, WU, B, BU):
        return (C * R.act(X @ W.t() + B, act) * (X @ WU.t() + BU)).sum()

    def differences(fn, args, at):
        out = torch.zeros_like(args[at]).reshape(-1)
        for e in range(out.numel()):
            lo, hi = ([t.clone() for t in args] for _ in range(2))
            lo[at].view(-1)[e] -= h
            hi[at].view(-1)[e] += h
            out[e] = (fn(*hi) - fn(*lo)) / (2 * h)
        return out.reshape(args[at].shape)

    for at, v in zip((0, 1, 2), got):
        torch.testing.assert_close(R.d(v), differences(loss, [X, W, B], at), rtol=2e-5, atol=2e-5)
    for at, v in zip((0, 1, 2, 3, 4), got_gated):
        torch.testing.assert_close(R.d(v), differences(gated_loss, [X, W, WU, B, BU], at), rtol=2e-5, atol=2e-5)


def test_binding_refusals(gpu_lib):
    import torch
    log("refusals")
    x, w, b, dy = make("bf16", 19, ((6, 24), 1.0), ((40, 24), 0.2), ((40,), 0.3), ((6, 40), 1.0))
    f = gpu_lib
    for call in (lambda: f.linear(x.float(), w), lambda: f.linear(x, w[:, :23]), lambda: f.linear(x, w, b[:39]),
                 lambda: f.linear(x, w, b.float()), lambda: f.linear(x, w, b, dy[:5]), lambda: f.linear(x.cpu(), w),
                 lambda: f.linear(x, w.cpu()), lambda: f.linear(x, w, activation="tanh"), lambda: f.linear(x, w, activation=3),
                 lambda: f.linear(x.double(), w.double()), lambda: f.linear(x.t(), w), lambda: f.linear(x[0], w),
                 lambda: f.linear(x[:1].expand(6, 24), w), lambda: f.linear(x[:, ::2], w[:, ::2]),
                 lambda: f.linear(x, w, out=dy.float()), lambda: f.linear(x, w, out=dy[:, :39]),
                 lambda: f.linear(x, w, b[::2].repeat_interleave(2)[::1][:39]), lambda: f.linear(x, None),
                 lambda: f.linear_backward(dy, x, w, activation="silu"), lambda: f.linear_backward(dy[:5], x, w),
                 lambda: f.gated_ffn(x, w, w[:39]), lambda: f.gated_ffn(x, w, w, b, b[:3]),
                 lambda: f.gated_ffn_backward(dy, x, w, w, dy, dy[:3]),
                 lambda: f.gated_ffn_backward(dy, x, w, w, dy, dy.half())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(embx_error(gpu_lib)):
        gpu_lib.linear(x[:, :0], w[:, :0])
    assert gpu_lib.linear(x, w).shape == (6, 40)


def embx_error(lib):
    return lib.EmbxError


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(64, 40, 64), (65, 40, 64), (65, 40, 65), (64, 40, 65), (66, 7, 32), (66, 7, 33), (200, 70, 64),
                                  (300, 513, 33), (64, 1000, 1000), (65, 1000, 1000), (1000, 24, 1)], ids=str)
def test_sizes_where_the_kernel_changes(gpu_lib, size, dtype):
    """Few rows or not, a short reduction or not, and one below or above."""
    m, n, k = size
    log(f"change of kernel {size} {dtype}")
    x, w, b, r = layer(dtype, 21, m, n, k, residual=True)
    wu, = make(dtype, 22, ((n, k), k ** -0.5))
    y, z = gpu_lib.linear(x, w, b, r, activation="gelu", save=True)
    for v, want in zip((y, z), R.linear(x, w, b, r, "gelu", dtype)):
        R.check(v, want, "linear")
    for v, want in zip(gpu_lib.gated_ffn(x, w, wu, b, None, save=True), R.gated(x, w, wu, b, None, "silu", dtype)):
        R.check(v, want, "gated")


@pytest.mark.parametrize("size", [(20, 24, 300), (150, 264, 200), (100, 24, 40)], ids=str)
def test_f32_at_the_ends_of_its_range(gpu_lib, size):
    """The largest numbers, against small ones so that the products are ordinary, and numbers of 2^-100: both are as
    accurate as any other."""
    import torch
    m, n, k = size
    log(f"range of f32 {size}")
    x, w, dy = make("f32", 23, ((m, k), 1.0), ((n, k), k ** -0.5), ((m, n), 1.0))
    x[:, 3] *= 2.0 ** 120
    x[1, 3] = torch.finfo(torch.float32).max
    x[2, 3] = -torch.finfo(torch.float32).max
    x[3, 3] = 2.0 ** 128 - 2.0 ** 119
    w[:, 3] *= 2.0 ** -126
    x[:, 4] *= 2.0 ** -100
    w[:, 4] *= 2.0 ** 100
    R.check(gpu_lib.linear(x, w), R.linear(x, w, None, None, "none", "f32")[0], "linear")
    wu = w.flip(0).contiguous()
    for v, want in zip(gpu_lib.gated_ffn(x, w, wu, activation="none", save=True), R.gated(x, w, wu, None, None, "none", "f32")):
        R.check(v, want, "gated")
    dx, dw, db = gpu_lib.linear_backward(dy, x * 2.0 ** -20, w)
    for v, want in zip((dx, dw, db), R.linear_backward(dy, x * 2.0 ** -20, w, None, "none", "f32")):
        R.check(v, want, "linear_backward")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(100, 72, 40), (65, 264, 64), (64, 40, 300), (1, 40, 300)], ids=str)
def test_infinities_and_nan_with_every_kernel(gpu_lib, size, dtype):
    """As above: only the results whose sums hold them, where there are few rows or the reduction is short."""
    import torch
    m, n, k = size
    log(f"not finite {size} {dtype}")
    x, w, dy, z = make(dtype, 24, ((m, k), 1.0), ((n, k), k ** -0.5), ((m, n), 0.5), ((m, n), 1.0))
    x[x == 0] = 0.5
    w[w == 0] = 0.5
    x[0, k - 1] = float("inf")
    x[m - 1, 5] = float("nan")
    for act in ("none", "relu"):
        want, got = R.linear(x, w, None, None, act, dtype)[0][0], R.d(gpu_lib.linear(x, w, activation=act))
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    # an infinite gradient behind a relu that is closed goes nowhere
    dy[0] = float("inf")
    z[0] = -1.0
    dx, dw, db = gpu_lib.linear_backward(dy, x.nan_to_num(1.0, 1.0), w, z, activation="relu")
    assert not R.d(dx)[0].any() and bool(torch.isfinite(R.d(dw)).all()) and bool(torch.isfinite(R.d(db)).all())


@pytest.mark.parametrize("size", [(300, 136, 520), (70, 8, 520), (20, 136, 520), (1100, 24, 40)], ids=str)
def test_every_kernel_beyond_32_bits(gpu_lib, size):
    """As above, with tiles, with few columns, with few rows and a short reduction: rows of x 2^23 bytes or more apart."""
    import torch
    m, n, k = size
    log(f"beyond 32 bits {size}")
    x, w, wu = make("f16", 25, ((m, k), 1.0), ((n, k), k ** -0.5), ((n, k), k ** -0.5))
    for ld in (1 << 22, (1 << 22) + 8):   # the second is more than the tiles take where it lies
        far = torch.empty_strided((m, k), (ld, 1), dtype=torch.float16, device="cuda")
        far.copy_(x)
        R.check(gpu_lib.linear(far, w), R.linear(x, w, None, None, "none", "f16")[0], "y")
        R.check(gpu_lib.gated_ffn(far, w, wu), R.gated(x, w, wu, None, None, "silu", "f16")[0], "h")
        del far


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(512, 256, 64), (512, 256, 72), (512, 384, 192), (1000, 200, 1030), (2048, 256, 128)], ids=str)
def test_tiles_in_halves(gpu_lib, size, dtype):
    """One step, an odd number of steps and a ragged last one, shared by the halves of a workgroup; both products of the
    gradients."""
    m, n, k = size
    log(f"halves {size} {dtype}")
    x, w, b, r = layer(dtype, 26, m, n, k, residual=True)
    dy, z = make(dtype, 27, ((m, n), 0.5), ((m, n), 1.0))
    wu, u = make(dtype, 28, ((n, k), k ** -0.5), ((m, n), 1.0))
    for v, want in zip(gpu_lib.linear(x, w, b, r, activation="relu", save=True), R.linear(x, w, b, r, "relu", dtype)):
        R.check(v, want, "linear")
    for v, want in zip(gpu_lib.gated_ffn(x, w, wu, None, b, save=True), R.gated(x, w, wu, None, b, "silu", dtype)):
        R.check(v, want, "gated")
    for v, want in zip(gpu_lib.linear_backward(dy, x, w, z, activation="silu"), R.linear_backward(dy, x, w, z, "silu", dtype)):
        R.check(v, want, "linear_backward")
    for v, want in zip(gpu_lib.gated_ffn_backward(dy, x, w, wu, z, u, bias=True), R.gated_backward(dy, x, w, wu, z, u, "silu", dtype)):
        R.check(v, want, "gated_backward")


def test_calls_keep_nothing(gpu_lib):
    """Neither memory nor references: results and workspace are the caller's or gone, after refusals too."""
    import sys

    import torch
    log("nothing kept")
    x, w, b, dy = make("f16", 29, ((70, 301), 1.0), ((90, 301), 0.1), ((90,), 0.3), ((70, 90), 1.0))
    out = torch.empty_like(dy)

    def calls():
        assert gpu_lib.linear(x, w, b, out=out) is out
        assert gpu_lib.linear(x, w, b, out=out, save=True)[0] is out
        assert gpu_lib.gated_ffn(x, w, w, b, out=out) is out
        gpu_lib.linear_backward(dy, x, w, dy, activation="silu")
        gpu_lib.gated_ffn_backward(dy, x, w, w, dy, dy, bias=True, need_dw=False)
        for bad in (lambda: gpu_lib.linear(x, w, b, activation=[]), lambda: gpu_lib.linear(x, w, dy)):
            with pytest.raises(ValueError):
                bad()

    calls()
    torch.cuda.synchronize()
    counts, memory = [sys.getrefcount(t) for t in (x, w, b, dy, out)], torch.cuda.memory_allocated()
    for _ in range(20):
        calls()
    assert [sys.getrefcount(t) for t in (x, w, b, dy, out)] == counts and torch.cuda.memory_allocated() == memory
    assert gpu_lib.linear(x, w, save=1)[1].shape == (70, 90)
