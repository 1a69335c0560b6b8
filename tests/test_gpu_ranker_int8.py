"""The example ranker with 8-bit weights: its scores are those of the same calls one by one, and each 8-bit layer is within its
bound of 64 bits on the inputs that it was given."""
import pytest

import dense_reference as R
import serving_reference as S
from gpu_helpers import log
from test_gpu_ranker import ranker  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("batch", [1, 100, 777])
def test_scores(gpu_lib, ranker, dtype, batch):  # noqa: F811
    import torch
    log(f"{dtype} {batch}")
    rows = [50, 3000, 700]
    r = ranker.make(rows, 64, batch, dtype)
    r.quantize()
    indices, offsets, dense, _ = ranker.queries(rows, batch, 1, dtype)
    got = r.scores(indices, offsets, dense, eight=True)
    p = r.p
    pooled = r.pooled(indices, offsets, batch)
    side = gpu_lib.linear(dense, p["wd"], p["bd"], activation="relu")
    x = gpu_lib.linear_int8(pooled, *r.eight["w0"], p["b0"], side, activation="relu")
    R.check(x, S.linear_int8(*S.quantize(pooled), *r.eight["w0"], p["b0"], side, "relu", dtype), "first layer")
    h = gpu_lib.gated_ffn(x, p["wg"], p["wu"])
    y = gpu_lib.linear_int8(h, *r.eight["wo"], p["bo"], x)
    R.check(y, S.linear_int8(*S.quantize(h), *r.eight["wo"], p["bo"], x, "none", dtype), "second layer")
    assert torch.equal(got, gpu_lib.linear(y, p["ws"], p["bs"], activation="sigmoid").view(-1))
    assert got.shape == (batch,) and got.dtype == r.dtype and bool(torch.isfinite(got).all())
