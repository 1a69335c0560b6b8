"""Every kernel of linear_int8 (the sizes of serving_kernels.py, which test_serving_choice.py holds to their kernels): whole
numbers exactly, results with everything that the epilogue does within their bounds, and nothing written outside of them."""
import pytest

import dense_reference as R
import serving_kernels as K
import serving_reference as S
from gpu_helpers import log

pytestmark = pytest.mark.gpu


def operands(case, seed):
    import torch
    m, n, k = case[1]
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def eights(*shape):
        return torch.randint(-128, 128, shape, generator=gen, device="cuda", dtype=torch.int8)

    def some(size, of):
        return of * (0.5 + torch.rand(size, generator=gen, device="cuda"))

    return eights(m, k), eights(n, k), some(m, 0.02), some(n, 0.02 * k ** -0.5), gen


@pytest.mark.parametrize("case", K.KERNELS, ids=K.name)
def test_whole_numbers(gpu_lib, case):
    import torch
    log(K.name(case))
    q, w, _, _, _ = operands(case, 1)
    m, n, _ = case[1]
    want = q.double() @ w.double().t()   # (exact in 64 bits in any order)
    y = gpu_lib.linear_int8(q, w, torch.ones(n, device="cuda"), x_scale=torch.ones(m, device="cuda"), dtype=torch.float32)
    assert torch.equal(y, want.float())
    assert torch.equal(y, gpu_lib.linear_int8(q, w, torch.ones(n, device="cuda"), x_scale=torch.ones(m, device="cuda"), dtype=torch.float32))


@pytest.mark.parametrize("case", K.KERNELS, ids=K.name)
def test_epilogue(gpu_lib, case):
    """Scales, bias, activation and residual, in a type for each case, into the residual inside a larger matrix of NaN."""
    import torch
    log(K.name(case))
    q, w, xs, ws, gen = operands(case, 2)
    m, n, k = case[1]
    dtype = ("f32", "f16", "bf16")[(m + k) % 3]
    bias = torch.randn(n, generator=gen, device="cuda").to(R.TYPES[dtype])
    around = torch.full((m + 2, n + 9), float("nan"), device="cuda", dtype=R.TYPES[dtype])
    out = around[1:-1, 4:4 + n]
    out.copy_(torch.randn(m, n, generator=gen, device="cuda"))
    r = out.clone()
    rows = torch.randperm(m, generator=gen, device="cuda")[:64]   # of which 64 bits are computed
    assert gpu_lib.linear_int8(q, w, ws, bias, out, x_scale=xs, activation="gelu", out=out) is out
    R.check(out[rows], S.linear_int8(q[rows], xs[rows], w, ws, bias, r[rows], "gelu", dtype), dtype)
    assert bool(torch.isfinite(out).all())
    out.fill_(float("nan"))
    assert bool(torch.isnan(around).all()), "written outside the result"
