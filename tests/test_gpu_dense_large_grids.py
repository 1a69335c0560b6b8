"""Layers of more outputs, or rows, than one workgroup for each 16 could be launched for: one query against 2^27 items, as
many queries of a narrow layer.  Operands are -1, 0 and 1: sums are exact."""
import pytest

from dense_reference import TYPES
from gpu_helpers import log

pytestmark = pytest.mark.gpu
PIECE = 1 << 24


def units(gen, dtype, rows, cols):
    import torch
    out = torch.empty((rows, cols), dtype=TYPES[dtype], device="cuda")
    for at in range(0, rows, PIECE):
        end = min(rows, at + PIECE)
        out[at:end] = torch.randint(-1, 2, (end - at, cols), generator=gen, dtype=torch.int8, device="cuda")
    return out


def test_one_query_many_items(gpu_lib):
    import torch
    n, k = (1 << 27) + 5, 128
    log(f"one query {n} {k}")
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w = units(gen, "f16", 1, k), units(gen, "f16", n, k)
    y = gpu_lib.linear(x, w)
    for at in range(0, n, PIECE):
        want = (x.float() @ w[at:at + PIECE].float().t()).half()
        assert torch.equal(y[:, at:at + PIECE], want), f"outputs from {at} on"


def test_many_rows_few_outputs(gpu_lib):
    import torch
    m, n, k = (1 << 28) + 3, 16, 72
    log(f"many rows {m} {n} {k}")
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, w = units(gen, "bf16", m, k), units(gen, "bf16", n, k)
    y = gpu_lib.linear(x, w)
    for at in range(0, m, PIECE):
        want = (x[at:at + PIECE].float() @ w.float().t()).bfloat16()
        assert torch.equal(y[at:at + PIECE], want), f"rows from {at} on"
