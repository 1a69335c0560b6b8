"""Which kernels moe_ffn takes: the sizes of moe_kernels.py take theirs, each kernel is among them (the GPU tests run them all), and
no size takes what its kernels cannot do."""
import ctypes
import math
import random

import pytest

import moe_kernels as K
import paper_2507_01676_amd as embx
from test_serving_arguments import FAKE, moe

DTYPES = {"f32": 0, "16": 2, "int8": 2}


def choose(kind, size, dtype=None):
    m, f, d, experts, top_k = size
    a = moe(FAKE if kind == "int8" else None, m=m, f=f, d=d, experts=experts, top_k=top_k,
            dtype=DTYPES[kind] if dtype is None else dtype, ldx=d, ldr=d, ldy=d, gate__ld=d, up__ld=d, down__ld=f)
    call = embx._lib["_ZN4embx10moe_chooseERK9emb_moe_t"]   # embx::moe_choose
    call.restype, call.argtypes = K.Choice, [ctypes.c_void_p]
    return call(ctypes.byref(a))


@pytest.mark.parametrize("kind,kernels,size", [(kind, *case) for kind, some in K.KERNELS.items() for case in some])
def test_kernels(kind, kernels, size):
    for dtype in {"f32": (0,), "16": (1, 2), "int8": (0, 1, 2)}[kind]:
        assert " | ".join(K.names(choose(kind, size, dtype), size[4])) == kernels


@pytest.mark.parametrize("kind", K.KERNELS)
def test_every_kernel(kind):
    parts = [tuple(name.split(" | ")) for name, _ in K.KERNELS[kind]]
    rows = ["16 rows", "32 rows"] + ["64 rows"] * (kind == "16")
    # a workgroup's wavefronts by what they multiply, and how many share it
    assert {", ".join(up.split(", ")[:2]) for _, up, _ in parts} == {f"{v}, {n} share" for v in ["4 columns", *rows] for n in (1, 2, 4, 8)}
    assert {up.split(",")[0] for _, up, _ in parts if up.endswith(", parts")} == {rows[-1]}   # (from 33 rows an expert on)
    # where it is found out which rows are whose
    have = {(routing, up.split(",")[0]) for routing, up, _ in parts}
    assert have == {(r, v) for r in ("route", "logits, route") for v in ["4 columns", *rows]} | {
        (r, v) for r in ("routing", "logits, routing") for v in ("4 columns", "16 rows")}
    by_rows = {"4 columns, 8 wavefronts", "4 columns, 16 wavefronts", "4 columns, 16 wavefronts, split",
               *("32 columns" + a + b for a in ("", ", split") for b in ("", ", few rows"))}
    blocks = {"f32": (16,), "16": (16, 32), "int8": ()}[kind]
    assert {down for _, _, down in parts} == by_rows | {f"by experts, {b} rows, {n} share{p}" for b in blocks for n in (1, 2, 4, 8)
                                                        for p in ("", ", parts")}


def test_limits():
    """Random layers within what is taken, the largest among them: lists, tables and grids hold them."""
    rng = random.Random(1)

    def size(most):
        return rng.choice([1, most, int(round(math.exp(rng.uniform(0, math.log(most)))))])

    for _ in range(20000):
        kind, experts = rng.choice(list(DTYPES)), size(1024)
        m, f, d, top_k = size(65536), size(1 << 25), size(1 << 25), size(min(experts, 32))
        c = choose(kind, (m, f, d, experts, top_k))
        what = (kind, m, f, d, experts, top_k)
        assert c.up_variant in (0, 1, 2) and c.down_variant in ((0, 1) if kind == "int8" else (0, 1, 2)), what
        assert c.up_waves in (1, 2, 4, 8) and 1 <= c.up_parts <= 256, what
        assert c.up_variant != 0 or m <= 4, what               # (rows that a lane has a place for)
        assert c.up_blocks == 2 or (c.up_blocks == 4 and kind == "16"), what
        if c.fused:                                             # the logits that a workgroup has room for
            assert c.up_variant < 2 and m * experts <= (256 if c.apart else 16), what
        assert not c.apart or m <= 256, what
        columns = (4 if c.up_variant == 0 else 16) * (8 // c.up_waves)
        assert -(-f // columns) * 512 < 1 << 32, what
        if c.down_variant == 2:
            assert c.down_waves in (1, 2, 4, 8) and c.down_blocks in ((1,) if kind == "f32" else (1, 2)) and c.splits == 1, what
            assert 1 <= c.down_parts <= 512 and m * top_k * d <= 1 << 26, what
        else:
            assert c.down_waves == 8 or (c.down_waves == 16 and c.down_variant == 0), what
            assert 1 <= c.down_rows <= 64 and c.down_rows * top_k <= 512 and 1 <= c.splits <= 16, what
            step = (64 if kind == "int8" else 32) * (4 if c.down_variant == 0 else 2)
            assert c.chunk % step == 0 and c.chunk >= step, what
            assert -(-d // (4 if c.down_variant == 0 else 32)) * c.down_waves * 64 < 1 << 32 and -(-m // c.down_rows) <= 65536, what
            assert c.splits == 1 or m * d < 1 << 32, what
