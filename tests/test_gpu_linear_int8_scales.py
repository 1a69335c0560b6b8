"""linear_int8 with scales far from one: what lies between a sum and a result that f32 holds is not too large for it."""
import pytest

import dense_reference as R
import serving_kernels as K
import serving_reference as S
from gpu_helpers import log

pytestmark = pytest.mark.gpu
# one size for each kernel
CASES = list({case[0]: case for case in K.KERNELS}.values())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=K.name)
def test_large_and_small_scales(gpu_lib, case, dtype):
    import torch
    log(f"{K.name(case)} {dtype}")
    m, n, k = case[1]
    gen = torch.Generator(device="cuda").manual_seed(m + k)
    q = torch.randint(-128, 128, (m, k), generator=gen, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (n, k), generator=gen, device="cuda", dtype=torch.int8)
    bias = torch.randn(n, generator=gen, device="cuda").to(R.TYPES[dtype])
    power = torch.tensor([125.0, -125.0, 97.0, 0.0, 110.0], device="cuda").repeat(m // 5 + 1)[:m]
    xs = 2.0 ** power * (0.5 + torch.rand(m, generator=gen, device="cuda"))
    rows = torch.randperm(m, generator=gen, device="cuda")[:60]
    for of in (125.0, 97.0, 0.0, -125.0):
        if m >= 5 or of == 125.0:
            near = 2.0 ** (-of - 6)   # of the weights' scales, for rows of that power
            ws = near * (0.5 + torch.rand(n, generator=gen, device="cuda"))
            take = rows[power[rows] == of] if m >= 5 else rows[:1]
            if len(take):
                y = gpu_lib.linear_int8(q, w, ws, bias, x_scale=xs, activation="none")
                value, bound = S.linear_int8(q[take], xs[take], w, ws, bias, None, "none", dtype)
                # (20000 products add up to 5 times 65504 here and there: f16 has the largest number for those, or an infinity)
                got, far = R.d(y[take]), value.abs() > torch.finfo(R.TYPES[dtype]).max
                assert bool((got.abs() >= torch.finfo(R.TYPES[dtype]).max)[far].all())
                R.check(torch.where(far, value, got), (value, bound), f"2^{of}")


@pytest.mark.parametrize("m", [1, 40])
def test_large_rows(gpu_lib, m):
    """Rows of f32 near its largest number, quantized on the way."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(m)
    x = (torch.rand(m, 512, generator=gen, device="cuda") - 0.5) * 6e38
    w = torch.randint(-128, 128, (70, 512), generator=gen, device="cuda", dtype=torch.int8)
    ws = 1e-36 * (0.5 + torch.rand(70, generator=gen, device="cuda"))
    want = S.linear_int8(*S.quantize(x), w, ws, None, None, "silu", "f32")
    R.check(gpu_lib.linear_int8(x, w, ws, activation="silu"), want, "large rows")
