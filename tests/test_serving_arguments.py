"""The serving forms' C entry points refuse what their header says they refuse, before they touch a device (these tests run
without one), and the workspace they ask for covers what they hold in it; the header compiles as C."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2507_01676_amd as embx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED = embx.ERR_INVALID_ARGUMENT, embx.ERR_UNSUPPORTED
FAKE = 1 << 20   # an aligned address that is never read: every call below is refused on the host
L, I, P = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p


def _struct(name, *fields):
    return type(name, (ctypes.Structure,), {"_fields_": list(fields)})


Quantize = _struct("emb_quantize_t", ("m", L), ("k", L), ("dtype", I), ("x", P), ("ldx", L), ("q", P), ("ldq", L), ("scale", P))
Linear = _struct("emb_linear_int8_t", ("m", L), ("n", L), ("k", L), ("dtype", I), ("activation", I), ("x", P), ("ldx", L),
                 ("x_scale", P), ("weight", P), ("ldw", L), ("w_scale", P), ("bias", P), ("residual", P), ("ldr", L), ("y", P),
                 ("ldy", L))
Experts = _struct("emb_experts_t", ("p", P), ("ld", L), ("stride", L), ("scale", P))
Moe = _struct("emb_moe_t", ("m", L), ("f", L), ("d", L), ("experts", I), ("top_k", I), ("dtype", I), ("activation", I),
              ("renormalize", I), ("x", P), ("ldx", L), ("router", P), ("ldr", L), ("gate", Experts), ("up", Experts),
              ("down", Experts), ("y", P), ("ldy", L), ("chosen", P), ("share", P))


def quantize(**changes):
    return _set(Quantize(24, 56, 2, FAKE, 56, FAKE, 56, FAKE), changes)


def linear(x_scale=FAKE, **changes):
    return _set(Linear(24, 40, 56, 2, 3, FAKE, 56, x_scale, FAKE, 56, FAKE, FAKE, FAKE, 40, FAKE, 40), changes)


def moe(scale=None, **changes):
    w = [Experts(FAKE, cols, 40 * 56, scale) for cols in (56, 56, 40)]
    return _set(Moe(24, 40, 56, 8, 2, 2, 3, 1, FAKE, 56, FAKE, 56, *w, FAKE, 56, FAKE, FAKE), changes)


def _set(a, changes):
    for name, v in changes.items():
        at, _, field = name.partition("__")
        if field:
            setattr(getattr(a, at), field, v)
        else:
            setattr(a, at, v)
    return a


def _bytes(a):
    return None if a is None else bytes(a)


def call(a, ws=FAKE, nbytes=1 << 60, name=None):
    if isinstance(a, Quantize):
        return embx._lib.emb_quantize(_bytes(a), None)
    name = name or ("emb_linear_int8" if isinstance(a, Linear) else "emb_moe")
    return getattr(embx._lib, name)(_bytes(a), ws, nbytes, None)


def size(a, name=None):
    n = ctypes.c_size_t(0)
    name = name or ("emb_linear_int8" if isinstance(a, Linear) else "emb_moe")
    code = getattr(embx._lib, name + "_workspace")(_bytes(a), ctypes.byref(n))
    return code, n.value


@pytest.mark.parametrize("changes,code", [
    ({"m": -1}, INVALID), ({"k": 0}, INVALID), ({"k": -3}, INVALID), ({"dtype": 3}, UNSUPPORTED), ({"dtype": -1}, UNSUPPORTED),
    ({"m": (1 << 30) + 1}, UNSUPPORTED), ({"k": (1 << 30) + 1}, UNSUPPORTED), ({"x": None}, INVALID), ({"q": None}, INVALID),
    ({"scale": None}, INVALID), ({"x": FAKE + 1}, INVALID), ({"scale": FAKE + 2}, INVALID), ({"ldx": 55}, INVALID),
    ({"ldq": 55}, INVALID), ({"ldx": -56}, INVALID), ({"ldx": (1 << 40) + 1}, UNSUPPORTED), ({"ldq": (1 << 40) + 1}, UNSUPPORTED)],
    ids=str)
def test_quantize(changes, code):
    assert call(quantize(**changes)) == code


def test_null_structs():
    assert embx._lib.emb_quantize(None, None) == INVALID
    for name, a in (("emb_linear_int8", linear()), ("emb_moe", moe())):
        assert call(None, name=name) == INVALID and size(None, name)[0] == INVALID
        assert getattr(embx._lib, name + "_workspace")(bytes(a), None) == INVALID


@pytest.mark.parametrize("changes,code", [
    ({"m": -1}, INVALID), ({"n": 0}, INVALID), ({"k": 0}, INVALID), ({"activation": -1}, INVALID), ({"activation": 5}, INVALID),
    ({"dtype": 3}, UNSUPPORTED), ({"m": (1 << 30) + 1}, UNSUPPORTED), ({"n": (1 << 30) + 1}, UNSUPPORTED),
    ({"k": 131072}, UNSUPPORTED), ({"m": 1 << 30, "n": 1 << 30}, UNSUPPORTED)], ids=str)
def test_linear_int8_shapes(changes, code):
    changes = {**changes, **({"ldx": 1 << 20, "ldw": 1 << 20} if "k" in changes else {}), **({"ldy": 1 << 30, "ldr": 1 << 30} if "n" in changes else {})}
    assert call(linear(**changes)) == code and size(linear(**changes))[0] == code


@pytest.mark.parametrize("changes,code", [
    ({"x": None}, INVALID), ({"weight": None}, INVALID), ({"w_scale": None}, INVALID), ({"y": None}, INVALID),
    ({"w_scale": FAKE + 1}, INVALID), ({"x_scale": FAKE + 2}, INVALID), ({"bias": FAKE + 1}, INVALID),
    ({"residual": FAKE + 1}, INVALID), ({"y": FAKE + 1}, INVALID), ({"ldx": 55}, INVALID), ({"ldw": 55}, INVALID),
    ({"ldr": 39}, INVALID), ({"ldy": 39}, INVALID), ({"ldy": -40}, INVALID), ({"ldw": (1 << 40) + 1}, UNSUPPORTED),
    ({"ldy": (1 << 40) + 1}, UNSUPPORTED), ({"x_scale": None, "x": FAKE + 1}, INVALID)], ids=str)
def test_linear_int8_operands(changes, code):
    assert call(linear(**changes)) == code


@pytest.mark.parametrize("changes,code", [
    ({"m": -1}, INVALID), ({"f": 0}, INVALID), ({"d": 0}, INVALID), ({"experts": 0}, INVALID), ({"top_k": 0}, INVALID),
    ({"top_k": 9}, INVALID), ({"activation": 5}, INVALID), ({"activation": -1}, INVALID), ({"dtype": 3}, UNSUPPORTED),
    ({"m": 65537}, UNSUPPORTED), ({"f": (1 << 25) + 1}, UNSUPPORTED), ({"d": (1 << 25) + 1}, UNSUPPORTED),
    ({"experts": 1025}, UNSUPPORTED), ({"experts": 64, "top_k": 33}, UNSUPPORTED), ({"gate__scale": FAKE}, INVALID),
    ({"up__scale": FAKE, "down__scale": FAKE}, INVALID)], ids=str)
def test_moe_shapes(changes, code):
    assert call(moe(**changes)) == code and size(moe(**changes))[0] == code


@pytest.mark.parametrize("scale", [None, FAKE])
@pytest.mark.parametrize("changes,code", [
    ({"x": None}, INVALID), ({"router": None}, INVALID), ({"y": None}, INVALID), ({"gate__p": None}, INVALID),
    ({"up__p": None}, INVALID), ({"down__p": None}, INVALID), ({"x": FAKE + 1}, INVALID), ({"router": FAKE + 1}, INVALID),
    ({"y": FAKE + 1}, INVALID), ({"chosen": FAKE + 2}, INVALID), ({"share": FAKE + 2}, INVALID), ({"ldx": 55}, INVALID),
    ({"ldr": 55}, INVALID), ({"ldy": 55}, INVALID), ({"gate__ld": 55}, INVALID), ({"up__ld": 55}, INVALID),
    ({"down__ld": 39}, INVALID), ({"gate__stride": -1}, INVALID), ({"down__ld": (1 << 25) + 1}, UNSUPPORTED),
    ({"up__stride": (1 << 40) + 1}, UNSUPPORTED), ({"ldx": (1 << 40) + 1}, UNSUPPORTED)], ids=str)
def test_moe_operands(scale, changes, code):
    assert call(moe(scale, **changes)) == code


def test_moe_scales_and_weights_alignment():
    assert call(moe(FAKE, gate__scale=FAKE + 1)) == INVALID
    assert call(moe(None, gate__p=FAKE + 1)) == INVALID


@pytest.mark.parametrize("x_scale", [None, FAKE])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (3, 4096, 12800), (24, 40, 56), (70000, 16, 24), (65536, 1024, 12800), (5, 70, 1001), (2050, 2050, 301)])
def test_linear_int8_workspace(x_scale, m, n, k):
    for ld, whole in ((k, k % 16 == 0), ((k + 15) // 16 * 16, True)):
        a = linear(x_scale, m=m, n=n, k=k, ldx=k, ldw=ld, ldr=n, ldy=n)
        code, need = size(a)
        assert code == embx.OK and need < 4 << 30
        padded = (k + 15) // 16 * 16
        if not whole and min(m, n) > 1000:
            assert need >= n * padded           # the weights' copy; the kernels of few rows or columns read them where they lie
        if x_scale is None and m > 8:
            assert need >= m * padded + 4 * m   # quantized x
        if need:
            assert call(a, FAKE, need - 1) == INVALID
            assert call(a, FAKE + 16, need) == INVALID
            assert call(a, None, need) == INVALID


@pytest.mark.parametrize("routing", [True, False])
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("m,f,d,experts,top_k", [(1, 1, 1, 1, 1), (5, 2816, 1024, 8, 2), (19, 333, 1001, 7, 3), (300, 40, 48, 64, 32)])
def test_moe_workspace(m, f, d, experts, top_k, dtype, routing):
    changes = dict(m=m, f=f, d=d, experts=experts, top_k=top_k, dtype=dtype, ldx=d, ldr=d, ldy=d, gate__ld=d, up__ld=d, down__ld=f)
    a = moe(None, **changes, **({} if routing else {"chosen": None, "share": None}))
    code, need = size(a)
    assert code == embx.OK
    assert need >= m * top_k * (4 * f + (0 if routing else 8))   # act(..) * (..) in 32 bits or twice 16, and the routing
    for ws, n in ((FAKE, need - 1), (FAKE + 16, need), (None, need)):
        assert call(a, ws, n) == INVALID


def test_no_rows_need_nothing():
    """With m == 0 matrices of no rows may be NULL, and nothing is launched."""
    assert call(quantize(m=0, x=None, q=None, scale=None)) == embx.OK
    a = linear(None, m=0, x=None, y=None, residual=None)
    assert size(a) == (embx.OK, 0) and call(a, None, 0) == embx.OK
    a = moe(None, m=0, x=None, y=None)
    assert size(a) == (embx.OK, 0) and call(a, None, 0) == embx.OK


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not available")
@pytest.mark.parametrize("lang", [["gcc", "-std=c99", "-pedantic", "-x", "c"], ["g++", "-std=c++17", "-x", "c++"]])
def test_header_compiles_and_agrees_with_the_structs(tmp_path, lang):
    structs = [Quantize, Linear, Experts, Moe]
    fields = "".join(f'  printf("%zu ", sizeof({s.__name__}));\n' for s in structs)
    src = tmp_path / "h.c"
    src.write_text(f'#include "embx_serving.h"\n#include <stdio.h>\nint main(void) {{\n{fields}  return 0;\n}}\n')
    exe = tmp_path / "h"
    r = subprocess.run([lang[0], *lang[1:], "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                        str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60).stdout
    assert [int(v) for v in out.split()] == [ctypes.sizeof(s) for s in structs]


def test_binding_refuses_host_tensors():
    import torch
    x, w, s = torch.zeros(3, 16), torch.zeros(5, 16, dtype=torch.int8), torch.zeros(5)
    e = torch.zeros(2, 8, 16)
    for call_ in (lambda: embx.quantize_rows(x), lambda: embx.linear_int8(x, w, s),
                  lambda: embx.moe_ffn(x, torch.zeros(2, 16), e, e, e.transpose(1, 2), top_k=1)):
        with pytest.raises(ValueError):
            call_()


def test_names():
    for name in ("quantize_rows", "linear_int8", "moe_ffn"):
        assert getattr(embx, name) is getattr(embx.serving, name) and name in dir(embx)


def test_package_without_the_binding():
    r = subprocess.run([os.sys.executable, "-c", "import sys; sys.modules['paper_2507_01676_amd._dense'] = None\n"
                        "import paper_2507_01676_amd as embx\n"
                        "for name in ('quantize_rows', 'linear_int8', 'moe_ffn'):\n"
                        "    try:\n        getattr(embx, name)\n"
                        "    except ImportError as e:\n        assert 'build it with' in str(e), e\n"
                        "    else:\n        raise SystemExit('no error from ' + name)\nprint('fine')"],
                       cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "fine" in r.stdout, r.stdout + r.stderr
