"""Which kernels a dense layer's call takes, and how its operands lie: the library's own entry points
(paper_2507_01676_amd/csrc/dense_api.cpp) compiled for the host with launches that only write down what they were given.
No device and no memory is touched."""
from __future__ import annotations

import ctypes
import functools
import os
import shutil
import subprocess
import tempfile

from test_dense_arguments import FAKE, OPS, _bytes

HERE = os.path.dirname(os.path.abspath(__file__))
CODES = {"f32": 0, "f16": 1, "bf16": 2}
ESIZE = {"f32": 4, "f16": 2, "bf16": 2}
TILE128, TILE256, HALVES, ROWS, SHORT = range(5)   # DenseVariant of csrc/dense.hpp
ROWS_OF = {"weight": "n", "w_gate": "n", "w_up": "n", "dweight": "n", "dw_gate": "n", "dw_up": "n"}      # others: m
COLS_OF = {k: "k" for k in ("x", "weight", "w_gate", "w_up", "dx", "dweight", "dw_gate", "dw_up")}       # others: n


def available():
    return shutil.which("g++") is not None


@functools.lru_cache(None)
def _lib():
    out = os.path.join(tempfile.mkdtemp(prefix="dense_launches_"), "launches.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "c", "dense_launches.cpp"), "-o", out],
                   check=True, capture_output=True, text=True)
    lib = ctypes.CDLL(out)
    lib.dense_launches.restype = ctypes.c_char_p
    for op in OPS:
        getattr(lib, op).argtypes = [ctypes.c_char_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        getattr(lib, op + "_workspace").argtypes = [ctypes.c_char_p, ctypes.POINTER(ctypes.c_size_t)]
    return lib


def launches(op, dtype, m, n, k, act=3, leave=(), **changes):
    """[(name, {field: value})] of a call with contiguous, aligned operands; ``leave``: operands that are not given (or
    wanted); ``changes``: fields set otherwise (a stride: ld_<operand>)."""
    sizes = {"m": m, "n": n, "k": k}
    a = OPS[op]()
    a.m, a.n, a.k, a.dtype, a.activation = m, n, k, CODES[dtype], act
    for name, _ in a._fields_[5:]:
        if name.startswith("ld_"):
            setattr(a, name, sizes[COLS_OF.get(name[3:], "n")])
        else:
            setattr(a, name, None if name in leave else FAKE)
    for name, v in changes.items():
        setattr(a, name, v)
    lib, need = _lib(), ctypes.c_size_t(0)
    code = getattr(lib, op + "_workspace")(_bytes(a), ctypes.byref(need))
    assert code == 0, f"{op} workspace: status {code}"
    lib.dense_launches()
    code = getattr(lib, op)(_bytes(a), FAKE, need.value, None)
    assert code == 0, f"{op}: status {code}"
    out = []
    for line in lib.dense_launches().decode().splitlines():
        name, *fields = line.split()
        out.append((name, {f.split("=")[0]: int(f.split("=")[1]) for f in fields}))
    return out


def products(*args, **kw):
    return [(name, f) for name, f in launches(*args, **kw) if name in ("forward", "dw", "dx")]
