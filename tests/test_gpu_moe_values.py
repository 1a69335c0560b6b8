"""Layers of experts where act(..) * (..) is small, large, or has bits that count: it is f32 with every type, all of the way."""
import pytest

import dense_reference as R
import moe_reference as M
from gpu_helpers import log
from test_gpu_serving import inside

pytestmark = pytest.mark.gpu

# rows, f, d, experts, top_k: by four columns and by 32, with parts of the reduction, by experts
SIZES = [(1, 96, 40, 4, 2), (2, 1000, 301, 3, 2), (20, 97, 41, 4, 2), (9, 2100, 72, 2, 1), (70, 501, 1101, 4, 1), (200, 300, 1100, 8, 1)]
ACTIVATIONS = ["none", "relu", "sigmoid", "silu", "gelu"]
KINDS = [(dtype, eight) for dtype in ("f32", "f16", "bf16") for eight in (False, True)]


def run(lib, o, act, dtype, what, **more):
    import torch
    y, chosen, share = lib.moe_ffn(o["x"], o["router"], *o["ws"], top_k=o["top_k"], scales=o["scales"], activation=act, routing=True, **more)
    want, experts, shares = M.moe(o["x"], o["router"], *o["ws"], o["top_k"], act, dtype, o["scales"])
    assert torch.equal(chosen.cpu(), experts)
    R.check(share, shares, "shares")
    R.check(y, want, what)
    # operands that start anywhere
    views = [inside(t, 5)[0] for t in (o["x"], o["router"], *o["ws"])]
    again = lib.moe_ffn(views[0], views[1], *views[2:], top_k=o["top_k"], scales=o["scales"], activation=act)
    R.check(again, want, what + ", of views")


@pytest.mark.parametrize("spread", M.SPREADS)
@pytest.mark.parametrize("dtype,eight", KINDS)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_all_bits_count(gpu_lib, size, dtype, eight, spread):
    log(f"moe values {size} {dtype} {eight} {spread}")
    run(gpu_lib, M.operands(size, dtype, 7, eight, spread, "cuda"), "none", dtype, spread)


@pytest.mark.parametrize("act", ACTIVATIONS)
@pytest.mark.parametrize("dtype,eight", KINDS)
@pytest.mark.parametrize("size", SIZES[:1] + SIZES[2:3] + SIZES[-1:], ids=str)
def test_activations(gpu_lib, size, dtype, eight, act):
    """Also far out, where the activations of negative values are small."""
    for seed, times in ((1, 0.5), (2, 4.0)):
        log(f"moe activations {size} {dtype} {eight} {act} {times}")
        o = M.operands(size, dtype, seed, eight, "even", "cuda")
        if eight:
            o["scales"] = (o["scales"][0] * times, *o["scales"][1:])
        else:
            o["ws"][0] *= times
        run(gpu_lib, o, act, dtype, f"{act} {times}")


@pytest.mark.parametrize("dtype,eight", KINDS)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_infinities(gpu_lib, size, dtype, eight):
    """An infinite act(..) * (..) gives infinities of its weights' signs, NaN where those are nought, and rows beside it nothing."""
    log(f"moe infinities {size} {dtype} {eight}")
    o = M.operands(size, dtype, 11, eight, "even", "cuda")
    at = size[1] // 2
    if eight:
        o["scales"][1][0, at] = float("inf")
    else:
        o["ws"][1][0, at] = float("inf") * o["x"].abs().amax(0).gt(0.5).to(o["x"].dtype)   # (nought elsewhere: not NaN)
        o["ws"][1][0, at].nan_to_num_(nan=0.0, posinf=float("inf"))
    down = o["ws"][2][0]
    down[::3, at] = 3
    down[1::3, at] = -2
    down[2::3, at] = 0
    run(gpu_lib, o, "none", dtype, "infinities")
