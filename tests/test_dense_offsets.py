"""Offsets within a tile of the dense layers' products stay below 2^31 bytes, for every length of a row that the entry
points take (host only: the kernels' launches are written down instead of made)."""
import pytest

import dense_launches as L

pytestmark = pytest.mark.skipif(not L.available(), reason="g++ not available")

# each of a tile's operands is addressed by 32-bit offsets from the tile's first element: of 256 rows where the reduction
# runs along the rows (128 in the smaller tiles), of a step of 64 where it runs across them
LONG = [("f32", 256, 256, 2200000), ("f32", 512, 512, 5000000), ("bf16", 512, 512, 5000000), ("bf16", 128, 128, 9000000),
        ("f16", 1024, 512, 5000000), ("f16", 300, 200, 100000000), ("f32", 512, 2200000, 64), ("f32", 256, 5000000, 256),
        ("bf16", 256, 9000000, 64), ("f16", 130, 40000000, 72), ("bf16", 2048, 300, 1 << 30), ("f32", 300, 1 << 30, 100)]


def check_strides(op, dtype, m, n, k, **kw):
    seen = 0
    for name, f in L.products(op, dtype, m, n, k, **kw):
        if f["variant"] in (L.ROWS, L.SHORT):   # 64-bit addresses
            continue
        seen += 1
        rows = 256 if f["variant"] == L.TILE256 else 128
        a_rows = rows if name in ("forward", "dx") else 64
        b_rows = rows if name == "forward" else 64
        strides = [(f["lda"], min(a_rows, f["ni"] if a_rows != 64 else f["nr"]))]
        for at in range(2 if (op.startswith("emb_gated") and name != "dw") else 1):
            strides.append((f[f"ldb{at}"], min(b_rows, f["nj"] if b_rows != 64 else f["nr"])))
        for ld, across in strides:
            last = (across - 1) * ld * L.ESIZE[dtype] + 256 * L.ESIZE[dtype]
            assert last < 1 << 31, f"{op} {name} {dtype} {m} x {n} x {k}: row {across - 1} of a tile starts {last} bytes on"
    return seen


@pytest.mark.parametrize("op", L.OPS)
@pytest.mark.parametrize("dtype,m,n,k", LONG)
def test_long_rows(op, dtype, m, n, k):
    seen = check_strides(op, dtype, m, n, k)
    assert seen or "backward" not in op
    if op == "emb_linear_backward":
        check_strides(op, dtype, m, n, k, act=0, leave=("z",))


@pytest.mark.parametrize("op,dtype,m,n,k", [
    ("emb_linear", "f32", 256, 256, 2200000), ("emb_gated", "bf16", 512, 260, 5000001), ("emb_linear", "f16", 700, 700, 700),
    ("emb_linear_backward", "f16", 300, 9000000, 40), ("emb_gated_backward", "f32", 300, 2200001, 40)])
def test_launches_cover_the_reduction(op, dtype, m, n, k):
    """Launches that share a reduction take all of it, and their partial sums lie one after another."""
    kind = "forward" if "backward" not in op else "dx"
    seen = [f for name, f in L.products(op, dtype, m, n, k) if name == kind]
    assert sum(f["nr"] for f in seen) == (n if kind == "dx" else k)
    first = 0
    for f in seen:
        assert f["first"] == first
        first += f["splits"]
    assert all(f["slots"] == first for f in seen)
    assert len([name for name, _ in L.products(op, dtype, m, n, k) if name == "dw"]) == (kind == "dx")


@pytest.mark.parametrize("op", L.OPS)
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_far_rows(op, dtype):
    """Short rows far apart, aligned or not."""
    names = [name for name, _ in L.OPS[op]._fields_ if name.startswith("ld_")]
    for ld in (1 << 21, (1 << 21) + 4, (1 << 22) + 8, (1 << 23) + 1, (1 << 40)):
        check_strides(op, dtype, 4096, 4096, 520, **{name: ld for name in names})
