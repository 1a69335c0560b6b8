"""No launch of the dense layers has 2^32 threads along an axis, which the runtime refuses, however many rows or outputs a
layer has (host only: the launches are written down instead of made)."""
import collections

import pytest

import dense_launches as L

pytestmark = pytest.mark.skipif(not L.available(), reason="g++ not available")

# as many as fit 288 GB: one query against the weights of 2^27 items and more, as many queries of small layers
SIZES = [("f16", 1, 1 << 27, 128), ("f32", 1, 1 << 28, 65), ("bf16", 17, 1 << 28, 66), ("f32", 1 << 29, 1, 72),
         ("f16", 1 << 30, 1, 100), ("f16", 1 << 28, 16, 100), ("bf16", 1 << 30, 8, 100), ("f32", 3, 1 << 30, 20),
         ("f32", 1, 1 << 30, 8), ("f32", 1 << 30, 1, 8), ("f16", 1 << 30, 40, 8), ("f32", 1 << 30, 40, 8),
         ("f16", 1, 1 << 30, 8),
         ("f16", 1 << 30, 40, 66), ("f32", 1 << 27, 200, 40), ("f16", 1 << 24, 4000, 40), ("bf16", 300000, 300000, 66)]


def threads(name, f, dtype):
    """along the grid's first axis"""
    if f["variant"] == L.ROWS:
        across, down = -(-f["nj"] // 16), -(-f["ni"] // (16 * f["row_blocks"]))
        return across * (down if down < 8 else -(-down // 8) * 8) * 512
    if f["variant"] == L.SHORT:
        return -(-f["nj"] // (128 if f["kind"] == 1 else 256)) * 256   # (or at most 1024 workgroups)
    wide = f["variant"] == L.TILE256
    rows, columns = 256 if wide else 128, 256 if wide and dtype != "f32" else 128
    tiles = -(-f["ni"] // rows) * -(-f["nj"] // (columns // 2 if f["kind"] == 1 else columns))
    if name == "dw":
        tiles = -(-tiles * f["splits"] * f["parts"] // 8) * 8
    elif name == "dx":
        tiles *= f["splits"]
    return tiles * (512 if dtype == "f32" or f["variant"] != L.TILE128 else 256)


@pytest.mark.parametrize("op", L.OPS)
@pytest.mark.parametrize("dtype,m,n,k", SIZES)
def test_threads_of_a_launch(op, dtype, m, n, k):
    of_call = collections.Counter()
    for name, f in L.products(op, dtype, m, n, k):
        of_call[f["call"]] += threads(name, f, dtype)
    assert of_call and max(of_call.values()) < 1 << 32, of_call
