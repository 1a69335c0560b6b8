"""Which kernel computes which dense layer: the sizes of dense_kernels.py take the kernels that they are listed under, and
among them is every kernel of every operator and type, split and not, with operands read where they lie and not.  A change
of the estimates behind the choice that moves a size to another kernel fails here (host only)."""
import pytest

import dense_kernels as K
import dense_launches as L

pytestmark = pytest.mark.skipif(not L.available(), reason="g++ not available")


def short_form(op, dtype, m, n, k):
    """wavefronts along columns, more than one chunk of rows (the launch's own arithmetic)"""
    wide = 32 if op == "gated" else 64
    waves = 1 if n <= wide else 2 if n <= 2 * wide else 4
    across, chunks = -(-n // (waves * wide)), -(-m // 64)
    most = 1024 if k <= 32 and dtype != "f32" else 512
    return waves, chunks > min(chunks, max(1, most // across))


@pytest.mark.parametrize("case", K.each(K.FORWARD), ids=K.name)
def test_forward(case):
    op, dtype, size, kernel, split, whole, form = case
    (_, f), = L.products("emb_" + op, dtype, *size)
    assert (f["variant"], f["splits"] > 1, bool(f["whole"])) == (kernel, split, whole)
    if kernel == L.ROWS:
        assert f["row_blocks"] == form
    if kernel == L.SHORT:
        assert short_form(op, dtype, *size) == form


@pytest.mark.parametrize("case", K.each(K.BACKWARD), ids=K.name)
def test_backward(case):
    op, dtype, size, kernel, w_split, x_split = case
    p = dict(L.products(f"emb_{op}_backward", dtype, *size))
    assert set(p) == {"dw", "dx"} and p["dw"]["variant"] == p["dx"]["variant"] == kernel
    assert (p["dw"]["splits"] > 1, p["dx"]["splits"] > 1) == (w_split, x_split)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("op", ["linear", "gated"])
def test_every_kernel_is_listed(op, dtype):
    seen = {tuple(c[3:]) for c in K.each(K.FORWARD) if c[:2] == (op, dtype)}
    tiles = (L.TILE128, L.TILE256) if dtype == "f32" else (L.TILE128, L.TILE256, L.HALVES)
    for tile in tiles:
        assert {s for k, s, _, _ in seen if k == tile} == {False, True}
        assert {w for k, s, w, _ in seen if k == tile and not s} == {False, True}
    assert {f for k, _, _, f in seen if k == L.ROWS} == {1, 2, 4}
    assert {w for k, _, w, _ in seen if k == L.ROWS} == {False, True}
    assert {f[0] for k, _, _, f in seen if k == L.SHORT} == {1, 2, 4}
    assert {(w, f[1]) for k, _, w, f in seen if k == L.SHORT} >= {(False, True), (True, True)}
    back = {tuple(c[3:]) for c in K.each(K.BACKWARD) if c[:2] == (op, dtype)}
    assert back == {(tile, w, x) for tile in tiles for w in (False, True) for x in (False, True)}
