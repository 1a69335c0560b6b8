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
