"""The serving forms where offsets pass 32 bits: rows, experts and results far apart, results of more than 2^31 elements, and
the most rows; and a graph of a layer of many experts."""
import pytest

import dense_reference as R
import serving_reference as S
from gpu_helpers import log
from test_gpu_serving import eights, generator, moe_operands, normal, some

pytestmark = pytest.mark.gpu


def far(t, stride):
    """The same values with rows (of matrices that follow one another, too) `stride` elements apart, in memory not cleared."""
    import torch
    n, k = t.shape[-2:]
    count = t.numel() // k
    base = torch.empty((count - 1) * stride + k, dtype=t.dtype, device="cuda")
    view = base.as_strided(t.shape, (*([n * stride] if t.dim() == 3 else []), stride, 1))
    view.copy_(t)
    return view


@pytest.mark.parametrize("dtype,k", [("bf16", 100), ("f16", 1001), ("f32", 20000)])
def test_quantize_rows_far_apart(gpu_lib, dtype, k):
    import torch
    gen = generator(k)
    x = normal(gen, dtype, 4, k)
    out = far(eights(gen, 4, k), (1 << 30) + 8), torch.empty(4, device="cuda")
    q, scale = gpu_lib.quantize_rows(far(x, (1 << 30) + 8), out=out)
    want, want_scale = S.quantize(x)
    assert torch.equal(R.d(q), want) and torch.equal(R.d(scale), want_scale)


@pytest.mark.parametrize("m,n,k,apart", [(5, 70, 200, 1 << 30), (5, 70, 201, (1 << 30) + 1), (700, 90, 200, 1 << 23), (700, 90, 256, (1 << 24) + 16)])
def test_linear_int8_rows_far_apart(gpu_lib, m, n, k, apart):
    import torch
    log(f"{m} {n} {k} {apart}")
    gen = generator(m)
    q, w, xs, ws = eights(gen, m, k), eights(gen, n, k), some(gen, m, of=0.02), some(gen, n, of=0.02 * k ** -0.5)
    r = normal(gen, "bf16", m, n)
    want = S.linear_int8(q, xs, w, ws, None, r, "silu", "bf16")
    fq, fw = far(q, apart), far(w, min(apart, 1 << 27))
    out = far(r, min(apart, (1 << 22) + 3))
    R.check(gpu_lib.linear_int8(fq, fw, ws, None, out, x_scale=xs, activation="silu", out=out), want, "x_scale")
    x = normal(gen, "bf16", m, k)
    y = gpu_lib.linear_int8(far(x, min(apart, 1 << 24)), fw, ws)
    assert torch.equal(y, gpu_lib.linear_int8(x, w, ws))


def test_linear_int8_large_result(gpu_lib):
    import torch
    m, n, k = 70000, 32000, 48   # 2.24e9 elements
    gen = generator(1)
    q, w, xs, ws = eights(gen, m, k), eights(gen, n, k), some(gen, m, of=0.02), some(gen, n, of=0.02)
    y = gpu_lib.linear_int8(q, w, ws, x_scale=xs, dtype=torch.bfloat16)
    rows = torch.tensor([0, 1, 33333, 67108, 67109, 69887, 69888, 69999], device="cuda")
    R.check(y[rows], S.linear_int8(q[rows], xs[rows], w, ws, None, None, "none", "bf16"), "rows")
    assert torch.equal(y[-200:], gpu_lib.linear_int8(q[-200:], w, ws, x_scale=xs[-200:], dtype=torch.bfloat16))


@pytest.mark.parametrize("dtype,eight,ld", [("bf16", False, 1 << 25), ("f32", False, (1 << 24) + 4), ("f16", True, (1 << 25) - 1)])
@pytest.mark.parametrize("m", [1, 9, 70])
def test_moe_far_apart(gpu_lib, m, dtype, eight, ld):
    """Experts' rows and experts as far apart as is taken, and rows of x and y beyond 2^31 bytes."""
    import torch
    log(f"{m} {dtype} {eight} {ld}")
    size = (m, 20, 40, 3, 2)
    o = moe_operands(size, dtype, m, eight)
    want, chosen, _ = S.moe(o["x"], o["router"], *o["ws"], 2, "silu", dtype, o["scales"])
    mats = [far(w, ld) for w in o["ws"]]
    apart = 1 << 30 if m == 1 else (1 << 31) // (m - 1)
    y, got, _ = gpu_lib.moe_ffn(far(o["x"], apart), far(o["router"], 1 << 28), *mats, top_k=2, scales=o["scales"], routing=True,
                                out=far(torch.empty_like(o["x"]), apart))
    assert torch.equal(got.cpu(), chosen)
    R.check(y, want, "experts")


@pytest.mark.parametrize("experts,top", [(8, 2), (40, 32)])
def test_moe_most_rows(gpu_lib, experts, top):
    import torch
    m = 65536
    o = moe_operands((m, 24, 40, experts, top), "bf16", top, False)
    y = gpu_lib.moe_ffn(o["x"], o["router"], *o["ws"], top_k=top)
    rows = torch.tensor([0, 1, 511, 512, 32767, 32768, 65000, 65535], device="cuda")
    want, _, _ = S.moe(o["x"][rows], o["router"], *o["ws"], top, "silu", "bf16")
    R.check(y[rows], want, "rows")
    assert bool(torch.isfinite(y).all())


@pytest.mark.parametrize("m", [2, 30])
def test_many_experts_captured_and_replayed(gpu_lib, m):
    import torch
    o = moe_operands((m, 64, 96, 48, 4), "bf16", m, False)
    gen = generator(m)
    gpu_lib.moe_ffn(o["x"], o["router"], *o["ws"], top_k=4)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = gpu_lib.moe_ffn(o["x"], o["router"], *o["ws"], top_k=4)
    for _ in range(4):
        o["x"].copy_(normal(gen, "bf16", m, 96))
        eager = gpu_lib.moe_ffn(o["x"], o["router"], *o["ws"], top_k=4)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager)
