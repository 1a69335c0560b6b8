"""The bounds of moe_reference hold results whose h is f32, and none whose h has been rounded: to the layer's type, to two values
of 16 bits, or to f16's range."""
import pytest
import torch

import dense_reference as R
import moe_reference as M

SIZE = (5, 96, 40, 4, 2)


def emulated(dtype, spread, eight, handed, act="none"):
    """R.check of what a layer gives whose h is handed on so"""
    o = M.operands(SIZE, dtype, 3, eight, spread)
    args = (o["x"], o["router"], *o["ws"], o["top_k"], act, dtype, o["scales"])
    want, _, _ = M.moe(*args)
    got, _, _ = M.moe(*args, handed=handed)
    R.check(got[0].to(R.TYPES[dtype]), want, "emulated")


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("spread", M.SPREADS)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_f32_is_within(dtype, spread, eight):
    for act in ("none", "relu", "sigmoid", "silu", "gelu"):
        emulated(dtype, spread, eight, lambda h, wd: (h, wd), act)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype,spread,handed", [
    ("f16", "even", M.f16_parts(1)), ("f16", "small", M.f16_parts(2)), ("f16", "large", M.f16_parts(2)), ("f16", "mixed", M.f16_parts(2)),
    ("f16", "even", M.bf16_parts(2)), *(("bf16", spread, M.bf16_parts(n)) for spread in M.SPREADS for n in (1, 2))])
def test_fewer_bits_are_not(dtype, spread, handed, eight):
    with pytest.raises(AssertionError, match="out of bounds|infinities|NaN"):
        emulated(dtype, spread, eight, handed)
