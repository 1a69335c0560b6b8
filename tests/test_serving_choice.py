"""Which kernel linear_int8 takes: the sizes of serving_kernels.py take theirs, and each kernel is among them (the GPU tests run
them all)."""
import ctypes

import pytest

import paper_2507_01676_amd as embx
import serving_kernels as K


class Choice(ctypes.Structure):
    _fields_ = [("variant", ctypes.c_int32), ("splits", ctypes.c_int32), ("row_blocks", ctypes.c_int32), ("row_columns", ctypes.c_int32)]


def choose(m, n, k, align, copied):
    f = embx._lib["_ZN4embx15dense_choose_i8Elllid"]   # embx::dense_choose_i8
    f.restype, f.argtypes = Choice, [ctypes.c_int64] * 3 + [ctypes.c_int, ctypes.c_double]
    c = f(m, n, k, align, copied)
    return c.variant, c.splits, c.row_blocks, c.row_columns


@pytest.mark.parametrize("case", K.KERNELS, ids=K.name)
def test_kernel(case):
    m, n, k = case[1]
    assert case[2] == (16 if k % 16 == 0 else 4 if k % 4 == 0 else 1)
    assert K.kernel(choose(m, n, k, case[2], K.copied(case)), m, n) == case[0]


def test_every_kernel():
    have = {c[0] for c in K.KERNELS}
    rows = {f"rows {f} {j}" for f in (1, 2, 4) for j in (1, 2)} | {f"rows {f} 1 by XCD" for f in (1, 2, 4)}
    tiles = {t + s for t in ("tile 128", "tile 256", "halves") for s in ("", " split")}
    assert have == rows | tiles
    for kernel in rows:
        assert {c[2] for c in K.KERNELS if c[0] == kernel} == {16, 4, 1}, kernel


def test_extreme_sizes():
    """No choice that a launch cannot have, and no more splits than the reduction has steps."""
    for m in (1, 1 << 20, 1 << 30):
        for n in (1, 4096, 1 << 30):
            for k in (1, 128, 131071):
                variant, splits, blocks, columns = choose(m, n, k, 16, 0)
                if variant < 0:
                    assert m * n > 1 << 32
                    continue
                assert 1 <= splits <= 128 and (splits == 1 or splits * 4 * 128 <= k + 127)
                assert (variant == 3) == (blocks in (1, 2, 4)) == (columns in (1, 2))
                if variant == 3:
                    assert 512 * -(-n // 16) * (-(-m // (16 * blocks)) + 8) <= (1 << 32) - 1
                else:
                    side = 256 if variant == 1 else 128
                    assert (256 if variant == 0 else 512) * -(-m // side) * -(-n // side) <= (1 << 32) - 1
