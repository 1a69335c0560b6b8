"""The dense layers' C entry points refuse what their header says they refuse, before they touch a device (these
tests run without one), and the workspace they ask for covers what they hold in it; the headers compile as C."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2507_01676_amd as embx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED = embx.ERR_INVALID_ARGUMENT, embx.ERR_UNSUPPORTED


def _struct(*fields):
    """A struct as the header lists it: sizes, type, activation, then matrices (name) and vectors (name ending in '.')."""
    out = [(f, ctypes.c_int64) for f in "mnk"] + [("dtype", ctypes.c_int32), ("activation", ctypes.c_int32)]
    for f in fields:
        out += [(f[:-1], ctypes.c_void_p)] if f.endswith(".") else [(f, ctypes.c_void_p), ("ld_" + f, ctypes.c_int64)]
    return type("Args", (ctypes.Structure,), {"_fields_": out})


OPS = {"emb_linear": _struct("x", "weight", "bias.", "residual", "y", "z"),
       "emb_linear_backward": _struct("dy", "x", "weight", "z", "dx", "dweight", "dbias."),
       "emb_gated": _struct("x", "w_gate", "w_up", "b_gate.", "b_up.", "h", "g", "u"),
       "emb_gated_backward": _struct("dh", "x", "w_gate", "w_up", "g", "u", "dx", "dw_gate", "dw_up", "db_gate.", "db_up.")}
M, N, K = 24, 40, 56
SHAPE_OF = {"x": (M, K), "weight": (N, K), "w_gate": (N, K), "w_up": (N, K), "dx": (M, K), "dweight": (N, K),
            "dw_gate": (N, K), "dw_up": (N, K)}          # all other matrices are [M, N]
OPTIONAL = {"emb_linear": {"bias", "residual", "z"}, "emb_linear_backward": {"dx", "dweight", "dbias"},
            "emb_gated": {"b_gate", "b_up", "g", "u"},
            "emb_gated_backward": {"dx", "dw_gate", "dw_up", "db_gate", "db_up"}}
FAKE = 1 << 20   # an aligned address that is never read: every call below is refused on the host


def good(op, **changes):
    a = OPS[op]()
    a.m, a.n, a.k, a.dtype, a.activation = M, N, K, 2, 3
    for name, _ in a._fields_[5:]:
        if name.startswith("ld_"):
            setattr(a, name, SHAPE_OF.get(name[3:], (M, N))[1])
        else:
            setattr(a, name, FAKE)
    for name, v in changes.items():
        setattr(a, name, v)
    return a


def _bytes(a):
    return None if a is None else bytes(a)


def size(op, a):
    n = ctypes.c_size_t(0)
    code = getattr(embx._lib, op + "_workspace")(_bytes(a), ctypes.byref(n))
    return code, n.value


def call(op, a, ws=FAKE, nbytes=1 << 60):
    return getattr(embx._lib, op)(_bytes(a), ws, nbytes, None)


@pytest.mark.parametrize("op", OPS)
def test_bad_sizes_types_and_activations(op):
    for change, code in [({"m": -1}, INVALID), ({"n": 0}, INVALID), ({"k": 0}, INVALID), ({"k": -5}, INVALID),
                         ({"activation": -1}, INVALID), ({"activation": 5}, INVALID), ({"dtype": 3}, UNSUPPORTED),
                         ({"dtype": -1}, UNSUPPORTED), ({"m": (1 << 30) + 1}, UNSUPPORTED), ({"n": 1 << 31}, UNSUPPORTED),
                         ({"k": 1 << 40}, UNSUPPORTED)]:
        assert call(op, good(op, **change)) == code, change
        assert size(op, good(op, **change))[0] == code, change
    assert call(op, None) == INVALID
    assert size(op, None)[0] == INVALID
    assert getattr(embx._lib, op + "_workspace")(bytes(good(op)), None) == INVALID


@pytest.mark.parametrize("op", OPS)
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_bad_pointers_and_strides(op, dtype):
    for name, _ in OPS[op]._fields_[5:]:
        if name.startswith("ld_"):
            cols = SHAPE_OF.get(name[3:], (M, N))[1]
            assert call(op, good(op, dtype=dtype, **{name: cols - 1})) == INVALID, name
            assert call(op, good(op, dtype=dtype, **{name: 0})) == INVALID, name
            assert call(op, good(op, dtype=dtype, **{name: -cols})) == INVALID, name
            assert call(op, good(op, dtype=dtype, **{name: (1 << 40) + 1})) == UNSUPPORTED, name
        else:
            assert call(op, good(op, dtype=dtype, **{name: FAKE + 1})) == INVALID, name
            if name not in OPTIONAL[op]:
                assert call(op, good(op, dtype=dtype, **{name: None})) == INVALID, name


@pytest.mark.parametrize("op", OPS)
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (3, 4096, 12800), (24, 40, 56), (70000, 16, 24), (65536, 1024, 12800)])
def test_workspace_checks(op, dtype, m, n, k):
    a = good(op, m=m, n=n, k=k, dtype=dtype)
    for name, _ in OPS[op]._fields_[5:]:
        if name.startswith("ld_"):
            setattr(a, name, max(n, k))
    code, need = size(op, a)
    assert code == embx.OK
    if need:
        assert call(op, a, FAKE, need - 1) == INVALID
        assert call(op, a, FAKE + 16, need) == INVALID
        assert call(op, a, None, need) == INVALID
    assert need < 4 << 30
    if op.endswith("backward"):
        # dz (dg and du) at least
        mats = 2 if "gated" in op else 1
        assert need >= mats * m * n * (4 if dtype == 0 else 2)


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not available")
@pytest.mark.parametrize("lang", [["gcc", "-std=c99", "-pedantic", "-x", "c"], ["g++", "-std=c++17", "-x", "c++"]])
def test_header_compiles_and_agrees_with_the_binding(tmp_path, lang):
    fields = "".join(f'  printf("%zu ", sizeof({t}));\n' for t in ("emb_linear_t", "emb_linear_grad_t", "emb_gated_t", "emb_gated_grad_t"))
    src = tmp_path / "h.c"
    src.write_text(f'#include "embx_dense.h"\n#include <stdio.h>\nint main(void) {{\n{fields}  return 0;\n}}\n')
    exe = tmp_path / "h"
    r = subprocess.run([lang[0], *lang[1:], "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                        str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60).stdout
    assert [int(v) for v in out.split()] == [ctypes.sizeof(s) for s in OPS.values()]


def test_binding_refuses_host_tensors():
    import torch
    x, w = torch.zeros(3, 4), torch.zeros(5, 4)
    for call_ in (lambda: embx.linear(x, w), lambda: embx.gated_ffn(x, w, w),
                  lambda: embx.linear_backward(torch.zeros(3, 5), x, w),
                  lambda: embx.gated_ffn_backward(torch.zeros(3, 5), x, w, w, torch.zeros(3, 5), torch.zeros(3, 5))):
        with pytest.raises(ValueError):
            call_()


def test_the_package_file_loads_under_another_name():
    """Beside the package, without being one: the lookup of another build of the library."""
    import importlib.util
    spec = importlib.util.spec_from_file_location("embx_other", embx.__file__)
    other = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(other)
    assert other.Plan is not embx.Plan and not hasattr(other, "linear") and hasattr(embx, "linear")
