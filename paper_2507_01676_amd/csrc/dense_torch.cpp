// The dense layers' calls and their serving forms' for Python: checks torch tensors, allocates results and workspace with
// torch's allocator and calls include/embx_dense.h and embx_serving.h on the current stream.  Argument marshalling only.
// It is compiled because a small call's time is the host's: 4.4 us with it, of which a launch is 2.6, and 7.1 with the same
// checks in Python.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <optional>
#include <stdexcept>
#include <string>

#include "../../include/embx_dense.h"
#include "../../include/embx_serving.h"

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
      if (code == EMB_OK && bytes == 0) {
        code = run(&s, nullptr, 0, stream);
      } else if (code == EMB_OK) {
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
Entry<emb_linear_int8_t> g_linear_int8 = {"emb_linear_int8", true};
Entry<emb_moe_t> g_moe = {"emb_moe", true};
emb_status_t (*g_quantize)(const emb_quantize_t*, void*) = nullptr;

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
  return t == at::kFloat ? "torch.float32" : t == at::kHalf ? "torch.float16" : t == at::kChar ? "torch.int8" : "torch.bfloat16";
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

  // eight: 8-bit integers are taken too; type_is() then names the call's type
  Common(PyObject* o, const char* name, bool eight = false) {
    if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda() || THPVariable_Unpack(o).dim() != 2)
      throw Refused(std::string(name) + " must be a 2-D device tensor");
    first = THPVariable_Unpack(o);
    type = first.scalar_type();
    if (!(eight && type == at::kChar)) type_is(type, name);
    device = first.get_device();
    if (device != c10::hip::current_device())
      throw Refused(std::string(name) + " is on cuda:" + std::to_string(device) + ", the current device is cuda:" +
                    std::to_string(c10::hip::current_device()));
    rows = first.size(0), cols = first.size(1);
    at = matrix(o, name, rows, cols);
  }

  void type_is(at::ScalarType t, const char* name) {
    type = t;
    if (type == at::kFloat) code = EMB_DTYPE_F32;
    else if (type == at::kHalf) code = EMB_DTYPE_F16;
    else if (type == at::kBFloat16) code = EMB_DTYPE_BF16;
    else throw Refused(std::string(name) + " must be float32, float16 or bfloat16, got " + at::toString(type));
  }

  std::string like(at::ScalarType t) const { return std::string(type_name(t)) + " tensor on cuda:" + std::to_string(device); }

  Matrix matrix(PyObject* o, const char* name, int64_t r, int64_t c) const { return matrix(o, name, r, c, type); }

  Matrix matrix(PyObject* o, const char* name, int64_t r, int64_t c, at::ScalarType type) const {
    if (!THPVariable_Check(o)) throw Refused(std::string(name) + " must be a 2-D " + like(type));
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != type || t.dim() != 2)
      throw Refused(std::string(name) + " must be a 2-D " + like(type));
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

  void* vector(PyObject* o, const char* name, int64_t n) const { return vector(o, name, n, type); }

  void* vector(PyObject* o, const char* name, int64_t n, at::ScalarType type) const {
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
    throw Refused(std::string(name) + " must be a contiguous [" + std::to_string(n) + "] " + like(type));
  }

  // matrices of all experts, and their scales, if they have any
  emb_experts_t experts(PyObject* o, const char* name, PyObject* scale, const char* scale_name, int64_t n, int64_t r, int64_t c) const {
    const at::ScalarType type = scale == Py_None ? this->type : at::kChar;
    if (!THPVariable_Check(o)) throw Refused(std::string(name) + " must be a 3-D " + like(type));
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != type || t.dim() != 3)
      throw Refused(std::string(name) + " must be a 3-D " + like(type));
    if (t.size(0) != n || t.size(1) != r || t.size(2) != c)
      throw Refused(std::string(name) + " must be [" + std::to_string(n) + ", " + std::to_string(r) + ", " + std::to_string(c) +
                    "], got [" + std::to_string(t.size(0)) + ", " + std::to_string(t.size(1)) + ", " + std::to_string(t.size(2)) + "]");
    if (recording && t.requires_grad()) refuse_gradient(name);
    if (t.is_neg()) refuse_negated(name);
    int64_t ld = t.stride(1);
    if ((t.stride(2) != 1 && c > 1) || (ld < c && r > 1))
      throw Refused(std::string(name) + " must have contiguous rows that do not overlap, got strides (" + std::to_string(t.stride(0)) +
                    ", " + std::to_string(ld) + ", " + std::to_string(t.stride(2)) + ")");
    emb_experts_t w = {t.data_ptr(), std::max(ld, c), n > 1 ? t.stride(0) : 0, nullptr};
    if (scale != Py_None) {
      if (THPVariable_Check(scale)) {
        const at::Tensor& s = THPVariable_Unpack(scale);
        if (s.is_cuda() && s.get_device() == device && s.scalar_type() == at::kFloat && s.dim() == 2 && s.size(0) == n &&
            s.size(1) == r && s.is_contiguous()) {
          if (recording && s.requires_grad()) refuse_gradient(scale_name);
          if (s.is_neg()) refuse_negated(scale_name);
          w.scale = static_cast<const float*>(s.data_ptr());
          return w;
        }
      }
      throw Refused(std::string(scale_name) + " must be a contiguous [" + std::to_string(n) + ", " + std::to_string(r) + "] " +
                    like(at::kFloat));
    }
    return w;
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

// x, q, scale (both or none: results)
PyObject* quantize(PyObject*, Args a, Py_ssize_t count) {
  return guarded(count, 3, [&]() -> PyObject* {
    const Common c(a[0], "x");
    const int64_t m = c.rows, k = c.cols;
    const bool given = a[1] != Py_None || a[2] != Py_None;
    Matrix q;
    at::Tensor made_q, made_scale;
    float* scale;
    if (given) {
      if (a[2] == Py_None) throw Refused("out must be a pair of tensors, q and scale");
      q = c.matrix(a[1], "q", m, k, at::kChar);
      scale = static_cast<float*>(c.vector(a[2], "scale", m, at::kFloat));
    } else {
      const int64_t ld = (k + 15) / 16 * 16;
      made_q = at::empty({m, ld}, c.first.options().dtype(at::kChar));
      if (ld != k) made_q = made_q.narrow(1, 0, k);
      made_scale = at::empty({m}, c.first.options().dtype(at::kFloat));
      q = {made_q.data_ptr(), ld}, scale = static_cast<float*>(made_scale.data_ptr());
    }
    const emb_quantize_t s = {m, k, c.code, c.at.p, c.at.ld, static_cast<int8_t*>(q.p), q.ld, scale};
    const emb_status_t code = g_quantize(&s, c10::hip::getCurrentHIPStream(c.first.get_device()).stream());
    if (code != EMB_OK) throw Failed{"emb_quantize", code};
    if (given) made_q = written(a[1]), made_scale = written(a[2]);
    return wrap_all(std::optional<at::Tensor>(made_q), std::optional<at::Tensor>(made_scale));
  });
}

// x, weight, w_scale, bias, residual, x_scale, activation, dtype, out
PyObject* linear_int8(PyObject*, Args a, Py_ssize_t count) {
  return guarded(count, 9, [&]() -> PyObject* {
    const int32_t act = activation(a[6]);
    const bool eight = a[5] != Py_None;
    Common c(a[0], "x", true);
    if (eight != (c.type == at::kChar))
      throw Refused(eight ? "x_scale is given: x must be int8" : "x is int8: x_scale must be given");
    if (a[7] != Py_None) {
      if (!THPDtype_Check(a[7])) throw Refused("dtype must be a torch.dtype, got " + text(PyObject_Repr(a[7])));
      const at::ScalarType type = reinterpret_cast<THPDtype*>(a[7])->scalar_type;
      if (!eight && type != c.type) throw Refused(std::string("dtype must be x's, ") + type_name(c.type));
      c.type_is(type, "dtype");
    } else if (eight) {
      PyObject* const like = a[8] != Py_None ? a[8] : a[4] != Py_None ? a[4] : a[3];
      c.type_is(THPVariable_Check(like) ? THPVariable_Unpack(like).scalar_type() : at::kBFloat16, "dtype");
    }
    const int64_t m = c.rows, k = c.cols, n = rows_of(a[1], "weight");
    const Matrix w = c.matrix(a[1], "weight", n, k, at::kChar), r = c.optional(a[4], "residual", m, n);
    if (a[2] == Py_None) throw Refused("w_scale must be a contiguous [" + std::to_string(n) + "] " + c.like(at::kFloat));
    const float* ws = static_cast<const float*>(c.vector(a[2], "w_scale", n, at::kFloat));
    const float* xs = static_cast<const float*>(c.vector(a[5], "x_scale", m, at::kFloat));
    void* bias = c.vector(a[3], "bias", n);
    const bool given = a[8] != Py_None;
    Matrix y;
    at::Tensor made;
    if (given) {
      y = c.matrix(a[8], "out", m, n);
    } else {
      made = at::empty({m, n}, c.first.options().dtype(c.type));
      y = {made.data_ptr(), n};
    }
    g_linear_int8({m, n, k, c.code, act, c.at.p, c.at.ld, xs, static_cast<const int8_t*>(w.p), w.ld, ws, bias, r.p, r.ld, y.p, y.ld},
                  c.first);
    if (!given) return THPVariable_Wrap(made);
    written(a[8]);
    Py_INCREF(a[8]);
    return a[8];
  });
}

// x, router, w_gate, w_up, w_down, top_k, s_gate, s_up, s_down, activation, renormalize, out, routing
PyObject* moe(PyObject*, Args a, Py_ssize_t count) {
  return guarded(count, 13, [&]() -> PyObject* {
    const int32_t act = activation(a[9]);
    const Common c(a[0], "x");
    const int64_t m = c.rows, d = c.cols, e = rows_of(a[1], "router");
    const Matrix router = c.matrix(a[1], "router", e, d);
    const long top = PyLong_Check(a[5]) ? PyLong_AsLong(a[5]) : -1;
    PyErr_Clear();
    if (top < 1 || top > e)
      throw Refused("top_k must be a whole number from 1 to the experts' " + std::to_string(e) + ", got " + text(PyObject_Repr(a[5])));
    if (!THPVariable_Check(a[2]) || THPVariable_Unpack(a[2]).dim() != 3) throw Refused("w_gate must be a 3-D device tensor");
    const int64_t f = THPVariable_Unpack(a[2]).size(1);
    const bool eight = a[6] != Py_None;
    if (eight != (a[7] != Py_None) || eight != (a[8] != Py_None)) throw Refused("scales must be of all three matrices, or None");
    emb_moe_t s = {};
    s.m = m, s.f = f, s.d = d, s.experts = static_cast<int32_t>(e), s.top_k = static_cast<int32_t>(top);
    if (e > INT32_MAX) throw Failed{"emb_moe", EMB_ERR_UNSUPPORTED};
    s.dtype = c.code, s.activation = act, s.renormalize = flag(a[10]);
    s.x = c.at.p, s.ldx = c.at.ld, s.router = router.p, s.ldr = router.ld;
    s.gate = c.experts(a[2], "w_gate", a[6], "scales[0]", e, f, d);
    s.up = c.experts(a[3], "w_up", a[7], "scales[1]", e, f, d);
    s.down = c.experts(a[4], "w_down", a[8], "scales[2]", e, d, f);
    const bool given = a[11] != Py_None, routing = flag(a[12]);
    at::Tensor made;
    if (given) {
      const Matrix y = c.matrix(a[11], "out", m, d);
      s.y = y.p, s.ldy = y.ld;
    } else {
      made = c.empty(m, d);
      s.y = made.data_ptr(), s.ldy = d;
    }
    std::optional<at::Tensor> chosen, share;
    if (routing) {
      chosen = at::empty({m, top}, c.first.options().dtype(at::kInt));
      share = at::empty({m, top}, c.first.options().dtype(at::kFloat));
      s.chosen = static_cast<int32_t*>(chosen->data_ptr()), s.share = static_cast<float*>(share->data_ptr());
    }
    g_moe(s, c.first);
    if (given) made = written(a[11]);
    if (routing) return wrap_all(std::optional<at::Tensor>(made), chosen, share);
    if (!given) return THPVariable_Wrap(made);
    Py_INCREF(a[11]);
    return a[11];
  });
}

// addresses of the library's functions: emb_quantize, then the others, each call and its workspace
PyObject* bind_serving(PyObject*, PyObject* args) {
  unsigned long long p[5];
  if (!PyArg_ParseTuple(args, "(KKKKK)", p, p + 1, p + 2, p + 3, p + 4)) return nullptr;
  g_quantize = reinterpret_cast<decltype(g_quantize)>(p[0]);
  g_linear_int8.run = reinterpret_cast<decltype(g_linear_int8.run)>(p[1]);
  g_linear_int8.size = reinterpret_cast<decltype(g_linear_int8.size)>(p[2]);
  g_moe.run = reinterpret_cast<decltype(g_moe.run)>(p[3]);
  g_moe.size = reinterpret_cast<decltype(g_moe.size)>(p[4]);
  Py_RETURN_NONE;
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
                           {"bind_serving", bind_serving, METH_VARARGS, nullptr},
                           {"quantize", method(quantize), METH_FASTCALL, nullptr},
                           {"linear_int8", method(linear_int8), METH_FASTCALL, nullptr},
                           {"moe", method(moe), METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_dense", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__dense() { return PyModule_Create(&g_module); }
