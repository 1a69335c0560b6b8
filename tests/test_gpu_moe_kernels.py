"""Every kernel of moe_ffn (the sizes of moe_kernels.py, which test_moe_choice.py holds to their kernels), with rows that start at
multiples of 16 bytes and anywhere: results and routing within their bounds, and nothing written outside of them."""
import pytest

import dense_reference as R
import moe_kernels as K
import moe_reference as M
from gpu_helpers import log
from test_gpu_serving import inside

pytestmark = pytest.mark.gpu

CASES = [(dtype, kind, kernels, size) for kind, some in K.KERNELS.items() for kernels, size in some
         for dtype in {"f32": ["f32"], "16": ["f16", "bf16"], "int8": ["f32", "f16", "bf16"]}[kind]]


def padded(t):
    """The same values, rows at multiples of 16 bytes, with other values behind them."""
    import torch
    n = t.shape[-1]
    big = torch.full((*t.shape[:-1], (n + 15) // 16 * 16), 77, dtype=t.dtype, device="cuda")
    big[..., :n] = t
    return big[..., :n]


@pytest.mark.parametrize("dtype,kind,kernels,size", CASES, ids=lambda v: str(v).replace(" ", ""))
def test_kernel(gpu_lib, dtype, kind, kernels, size):
    import torch
    act = ("none", "silu", "gelu", "relu", "sigmoid")[sum(size) % 5]
    log(f"{dtype} {kind} {kernels} {size} {act}")
    o = M.operands(size, dtype, sum(size), kind == "int8", "even", "cuda")
    want, experts, shares = M.moe(o["x"], o["router"], *o["ws"], o["top_k"], act, dtype, o["scales"])
    for what, lay in (("whole", padded), ("anywhere", lambda t: inside(t, 5)[0])):
        x, router, *ws = [lay(t) for t in (o["x"], o["router"], *o["ws"])]
        out, around = inside(torch.zeros_like(o["x"]))
        y, chosen, share = gpu_lib.moe_ffn(x, router, *ws, top_k=o["top_k"], scales=o["scales"], activation=act, out=out, routing=True)
        assert y is out and torch.equal(chosen.cpu(), experts), what
        R.check(share, shares, what + ": shares")
        R.check(y, want, what)
        again = gpu_lib.moe_ffn(x, router, *ws, top_k=o["top_k"], scales=o["scales"], activation=act)
        assert torch.equal(again, y), what + ": equal calls, equal bits"
        out.fill_(float("nan"))
        assert bool(torch.isnan(around).all()), what + ": written outside the result"


@pytest.mark.parametrize("m", [32768, 32769])
def test_as_many_rows_as_partial_sums_fit_and_one_more(gpu_lib, m):
    """Results of each use, in f32, take memory: beyond 2^26 of them the down projection goes by rows again."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(m)
    log(f"{m} rows, 2 of 8 of 264 x 1024")

    def normal(*shape, std):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).bfloat16()

    x, router = normal(m, 1024, std=1.0), normal(8, 1024, std=2.0 / 32)
    ws = [normal(8, 264, 1024, std=1 / 32), normal(8, 264, 1024, std=1 / 32), normal(8, 1024, 264, std=1 / 16)]
    y, chosen, share = gpu_lib.moe_ffn(x, router, *ws, top_k=2, routing=True)
    rows = torch.tensor([0, 1, 63, 64, 511, 4095, 4096, 16384, 32700, 32766, 32767, m - 1], device="cuda")
    want, experts, shares = M.moe(x[rows], router, *ws, 2, "silu", "bf16")
    assert torch.equal(chosen[rows].cpu(), experts)
    R.check(share[rows], shares, "shares")
    R.check(y[rows], want, "rows")
    assert bool(torch.isfinite(y).all())
