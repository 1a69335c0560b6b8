// The dense layers' calls for Python: checks torch tensors, allocates results and workspace with torch's allocator and
// calls include/embx_dense.h on the current stream.  Argument marshalling only.  It is compiled because a small call's time
// is the host's: 4.4 us with it, of which a launch is 2.6, and 7.1 with the same checks in Python.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>
#include <stdexcept>
#include <string>

#include "../../include/embx_dense.h"

namespace {

// a refused argument: ValueError
struct Refused : std::runtime_error {
  using std::runtime_error::runtime_error;
};

// a call's status other than EMB_OK: the package's error
struct Failed {
  const char* name;
  emb_status_t code;
};

PyObject* g_error = nullptr;         // the package's error class
PyObject* g_activations = nullptr;   // names to codes

// An entry of the library and the size of its workspace.
template <class S>
struct Entry {
  const char* name;
  bool asks;   // most calls need a workspace: its size is asked for first, not after a refusal
  emb_status_t (*run)(const S*, void*, size_t, void*) = nullptr;
  emb_status_t (*size)(const S*, size_t*) = nullptr;

  void operator()(const S& s, const at::Tensor& x) const {
    void* stream = c10::hip::getCurrentHIPStream(x.get_device()).stream();
    emb_status_t code = asks ? EMB_ERR_INVALID_ARGUMENT : run(&s, nullptr, 0, stream);
    if (code == EMB_ERR_INVALID_ARGUMENT) {
      size_t bytes = 0;
      code = size(&s, &bytes);
      if (code == EMB_OK) {
        const at::Tensor ws = at::empty({static_cast<int64_t>(bytes)}, x.options().dtype(at::kByte));
        code = run(&s, ws.data_ptr(), bytes, stream);
      }
    }
    if (code != EMB_OK) throw Failed{name, code};
  }
};

Entry<emb_linear_t> g_linear = {"emb_linear", false};
Entry<emb_linear_grad_t> g_linear_backward = {"emb_linear_backward", true};
Entry<emb_gated_t> g_gated = {"emb_gated", false};
Entry<emb_gated_grad_t> g_gated_backward = {"emb_gated_backward", true};

std::string text(PyObject* repr) {
  const char* s = repr ? PyUnicode_AsUTF8(repr) : nullptr;
  std::string out = s ? s : "?";
  Py_XDECREF(repr);
  PyErr_Clear();
  return out;
}

int32_t activation(PyObject* name) {
  PyObject* code = PyDict_GetItemWithError(g_activations, name);
  if (code) return static_cast<int32_t>(PyLong_AsLong(code));
  PyErr_Clear();
  std::string names;
  PyObject *key, *value;
  for (Py_ssize_t at = 0; PyDict_Next(g_activations, &at, &key, &value);)
    names += (names.empty() ? "" : ", ") + std::string(PyUnicode_AsUTF8(key));
  throw Refused("activation must be one of " + names + ", got " + text(PyObject_Repr(name)));
}

const char* type_name(at::ScalarType t) {
  return t == at::kFloat ? "torch.float32" : t == at::kHalf ? "torch.float16" : "torch.bfloat16";
}

// The calls record nothing for torch's differentiation: a result would lack its gradient without a word.
[[gnu::noinline]] void refuse_gradient(const char* name) {
  throw Refused(std::string(name) + " requires a gradient, which this call does not record: call it under torch.no_grad() or "
                "in a torch.autograd.Function, or give " + name + ".detach(); the _backward functions compute the gradients");
}

[[gnu::noinline]] void refuse_negated(const char* name) {
  throw Refused(std::string(name) + " is a view that is negated when it is read: give " + name + ".resolve_neg()");
}

struct Matrix {
  void* p;
  int64_t ld;
};

// What the operands of a call have in common, from the one that the others are measured against.
struct Common {
  at::Tensor first;
  at::ScalarType type;
  int32_t code;
  int64_t device, rows, cols;
  const bool recording = c10::GradMode::is_enabled();
  Matrix at;

  Common(PyObject* o, const char* name) {
    if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda() || THPVariable_Unpack(o).dim() != 2)
      throw Refused(std::string(name) + " must be a 2-D device tensor");
    first = THPVariable_Unpack(o);
    type = first.scalar_type();
    if (type == at::kFloat) code = EMB_DTYPE_F32;
    else if (type == at::kHalf) code = EMB_DTYPE_F16;
    else if (type == at::kBFloat16) code = EMB_DTYPE_BF16;
    else throw Refused(std::string(name) + " must be float32, float16 or bfloat16, got " + at::toString(type));
    device = first.get_device();
    if (device != c10::hip::current_device())
      throw Refused(std::string(name) + " is on cuda:" + std::to_string(device) + ", the current device is cuda:" +
                    std::to_string(c10::hip::current_device()));
    rows = first.size(0), cols = first.size(1);
    at = matrix(o, name, rows, cols);
  }

  std::string like() const { return std::string(type_name(type)) + " tensor on cuda:" + std::to_string(device); }

  Matrix matrix(PyObject* o, const char* name, int64_t r, int64_t c) const {
    if (!THPVariable_Check(o)) throw Refused(std::string(name) + " must be a 2-D " + like());
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != type || t.dim() != 2)
      throw Refused(std::string(name) + " must be a 2-D " + like());
    if (t.size(0) != r || t.size(1) != c)
      throw Refused(std::string(name) + " must be [" + std::to_string(r) + ", " + std::to_string(c) + "], got [" +
                    std::to_string(t.size(0)) + ", " + std::to_string(t.size(1)) + "]");
    if (recording && t.requires_grad()) refuse_gradient(name);
    if (t.is_neg()) refuse_negated(name);
    int64_t ld = t.stride(0);
    if (t.stride(1) != 1 && c > 1)
      throw Refused(std::string(name) + " must have contiguous rows, got strides (" + std::to_string(ld) + ", " +
                    std::to_string(t.stride(1)) + ")");
    if (ld < c) {
      if (r > 1) throw Refused(std::string(name) + ": rows must not overlap, got a stride of " + std::to_string(ld));
      ld = c;
    }
    return {t.data_ptr(), ld};
  }

  Matrix optional(PyObject* o, const char* name, int64_t r, int64_t c) const {
    return o == Py_None ? Matrix{nullptr, 0} : matrix(o, name, r, c);
  }

  void* vector(PyObject* o, const char* name, int64_t n) const {
    if (o == Py_None) return nullptr;
    if (THPVariable_Check(o)) {
      const at::Tensor& t = THPVariable_Unpack(o);
      if (t.is_cuda() && t.get_device() == device && t.scalar_type() == type && t.dim() == 1 && t.size(0) == n &&
          (n == 1 || t.stride(0) == 1)) {
        if (recording && t.requires_grad()) refuse_gradient(name);
        if (t.is_neg()) refuse_negated(name);
        return t.data_ptr();
      }
    }
    throw Refused(std::string(name) + " must be a contiguous [" + std::to_string(n) + "] " + like());
  }

  at::Tensor empty(int64_t r, int64_t c) const { return at::empty({r, c}, first.options()); }
  at::Tensor empty(int64_t n) const { return at::empty({n}, first.options()); }
};

int64_t rows_of(PyObject* o, const char* name) {
  if (!THPVariable_Check(o) || THPVariable_Unpack(o).dim() != 2) throw Refused(std::string(name) + " must be a 2-D device tensor");
  return THPVariable_Unpack(o).size(0);
}

PyObject* wrap(const std::optional<at::Tensor>& t) {
  if (t) return THPVariable_Wrap(*t);
  Py_RETURN_NONE;
}

template <class... T>
PyObject* wrap_all(const T&... t) {
  PyObject* out = PyTuple_New(sizeof...(t));
  if (!out) return nullptr;
  Py_ssize_t n = 0;
  for (PyObject* o : {wrap(t)...}) {
    if (!o) {
      Py_DECREF(out);
      return nullptr;
    }
    PyTuple_SET_ITEM(out, n++, o);
  }
  return out;
}

bool flag(PyObject* o) {
  const int is = PyObject_IsTrue(o);
  if (is < 0) throw python_error();
  return is;
}

// A tensor given for the result, which now holds it: it counts as changed (one made in inference mode has no count).
at::Tensor written(PyObject* o) {
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
  return t;
}

void* pointer(const std::optional<at::Tensor>& t) { return t ? t->data_ptr() : nullptr; }

// body() with C++'s exceptions as Python's
template <class F>
PyObject* guarded(Py_ssize_t have, Py_ssize_t want, F body) {
  HANDLE_TH_ERRORS
  if (have != want) {
    PyErr_Format(PyExc_TypeError, "takes %zd arguments, got %zd", want, have);
    return nullptr;
  }
  try {
    return body();
  } catch (const Refused& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const Failed& e) {
    PyObject* args = Py_BuildValue("(is)", static_cast<int>(e.code), e.name);
    if (args) {
      PyErr_SetObject(g_error, args);
      Py_DECREF(args);
    }
  }
  return nullptr;
  END_HANDLE_TH_ERRORS
}

using Args = PyObject* const*;

// x, weight, bias, residual, activation, out, save
PyObject* linear(PyObject*, Args a, Py_ssize_t count) {
  return guarded(count, 7, [&]() -> PyObject* {
    const int32_t act = activation(a[4]);
    const Common c(a[0], "x");
    const int64_t m = c.rows, k = c.cols, n = rows_of(a[1], "weight");
    const Matrix w = c.matrix(a[1], "weight", n, k), r = c.optional(a[3], "residual", m, n);
    void* bias = c.vector(a[2], "bias", n);
    const bool given = a[5] != Py_None, save = flag(a[6]);
    Matrix y;
    at::Tensor made;
    if (given) {
      y = c.matrix(a[5], "out", m, n);
    } else {
      made = c.empty(m, n);
      y = {made.data_ptr(), n};
    }
    std::optional<at::Tensor> z;
    if (save) z = c.empty(m, n);
    g_linear({m, n, k, c.code, act, c.at.p, c.at.ld, w.p, w.ld, bias, r.p, r.ld, y.p, y.ld, pointer(z), save ? n : 0}, c.first);
    if (given) made = written(a[5]);
    if (!save && given) {
      Py_INCREF(a[5]);
      return a[5];
    }
    return save ? wrap_all(std::optional<at::Tensor>(made), z) : THPVariable_Wrap(made);
  });
}

// dy, x, weight, z, activation, bias, need_dx, need_dw
PyObject* linear_backward(PyObject*, Args a, Py_ssize_t count) {
  return guarded(count, 8, [&]() -> PyObject* {
    const int32_t act = activation(a[4]);
    const Common c(a[1], "x");
    const int64_t m = c.rows, k = c.cols, n = rows_of(a[2], "weight");
    if (act != EMB_ACT_NONE && a[3] == Py_None)
      throw Refused("activation " + text(PyObject_Repr(a[4])) + " needs z, the sums that linear(..., save=True) returns");
    const Matrix dy = c.matrix(a[0], "dy", m, n), w = c.matrix(a[2], "weight", n, k);
    const Matrix z = act != EMB_ACT_NONE ? c.matrix(a[3], "z", m, n) : Matrix{nullptr, 0};
    std::optional<at::Tensor> dx, dw, db;
    if (flag(a[6])) dx = c.empty(m, k);
    if (flag(a[7])) dw = c.empty(n, k);
    if (flag(a[5])) db = c.empty(n);
    g_linear_backward({m, n, k, c.code, act, dy.p, dy.ld, c.at.p, c.at.ld, w.p, w.ld, z.p, z.ld, pointer(dx), k, pointer(dw), k,
                       pointer(db)}, c.first);
    return wrap_all(dx, dw, db);
  });
}

// x, w_gate, w_up, b_gate, b_up, activation, out, save
PyObject* gated(PyObject*, Args a, Py_ssize_t count) {
  return guarded(count, 8, [&]() -> PyObject* {
    const int32_t act = activation(a[5]);
    const Common c(a[0], "x");
    const int64_t m = c.rows, k = c.cols, n = rows_of(a[1], "w_gate");
    const Matrix wg = c.matrix(a[1], "w_gate", n, k), wu = c.matrix(a[2], "w_up", n, k);
    void *bg = c.vector(a[3], "b_gate", n), *bu = c.vector(a[4], "b_up", n);
    const bool given = a[6] != Py_None, save = flag(a[7]);
    Matrix h;
    at::Tensor made;
    if (given) {
      h = c.matrix(a[6], "out", m, n);
    } else {
      made = c.empty(m, n);
      h = {made.data_ptr(), n};
    }
    std::optional<at::Tensor> g, u;
    if (save) g = c.empty(m, n), u = c.empty(m, n);
    const int64_t ld = save ? n : 0;
    g_gated({m, n, k, c.code, act, c.at.p, c.at.ld, wg.p, wg.ld, wu.p, wu.ld, bg, bu, h.p, h.ld, pointer(g), ld, pointer(u), ld},
            c.first);
    if (given) made = written(a[6]);
    if (!save && given) {
      Py_INCREF(a[6]);
      return a[6];
    }
    return save ? wrap_all(std::optional<at::Tensor>(made), g, u) : THPVariable_Wrap(made);
  });
}

// dh, x, w_gate, w_up, g, u, activation, bias, need_dx, need_dw
PyObject* gated_backward(PyObject*, Args a, Py_ssize_t count) {
  return guarded(count, 10, [&]() -> PyObject* {
    const int32_t act = activation(a[6]);
    const Common c(a[1], "x");
    const int64_t m = c.rows, k = c.cols, n = rows_of(a[2], "w_gate");
    const Matrix dh = c.matrix(a[0], "dh", m, n), wg = c.matrix(a[2], "w_gate", n, k), wu = c.matrix(a[3], "w_up", n, k);
    const Matrix g = c.matrix(a[4], "g", m, n), u = c.matrix(a[5], "u", m, n);
    std::optional<at::Tensor> dx, dwg, dwu, dbg, dbu;
    if (flag(a[8])) dx = c.empty(m, k);
    if (flag(a[9])) dwg = c.empty(n, k), dwu = c.empty(n, k);
    if (flag(a[7])) dbg = c.empty(n), dbu = c.empty(n);
    g_gated_backward({m, n, k, c.code, act, dh.p, dh.ld, c.at.p, c.at.ld, wg.p, wg.ld, wu.p, wu.ld, g.p, g.ld, u.p, u.ld,
                      pointer(dx), k, pointer(dwg), k, pointer(dwu), k, pointer(dbg), pointer(dbu)}, c.first);
    return wrap_all(dx, dwg, dwu, dbg, dbu);
  });
}

// (addresses of the library's eight functions, each call and its workspace; the error class; activations)
PyObject* bind(PyObject*, PyObject* args) {
  unsigned long long p[8];
  PyObject *error, *activations;
  if (!PyArg_ParseTuple(args, "(KKKKKKKK)OO!", p, p + 1, p + 2, p + 3, p + 4, p + 5, p + 6, p + 7, &error, &PyDict_Type, &activations))
    return nullptr;
  auto take = [&](auto& entry, int at) {
    entry.run = reinterpret_cast<decltype(entry.run)>(p[at]);
    entry.size = reinterpret_cast<decltype(entry.size)>(p[at + 1]);
  };
  take(g_linear, 0), take(g_linear_backward, 2), take(g_gated, 4), take(g_gated_backward, 6);
  Py_INCREF(error);
  Py_INCREF(activations);
  Py_XSETREF(g_error, error);
  Py_XSETREF(g_activations, activations);
  Py_RETURN_NONE;
}

template <class F>
PyCFunction method(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef g_methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                           {"linear", method(linear), METH_FASTCALL, nullptr},
                           {"linear_backward", method(linear_backward), METH_FASTCALL, nullptr},
                           {"gated", method(gated), METH_FASTCALL, nullptr},
                           {"gated_backward", method(gated_backward), METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_dense", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__dense() { return PyModule_Create(&g_module); }
