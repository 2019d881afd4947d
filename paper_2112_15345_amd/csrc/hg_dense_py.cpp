// The dense operators for the Python binding (module _hgdense): tensors checked,
// outputs and workspaces made, and the library's entry point called in one native call.
// A call on one row takes some 5 us on the device; through ctypes structures and torch's
// Python functions its marshalling took 12 to 15.
//
// Every function takes tensors (or None) and plain values, works on the tensors' device
// and the current stream, and returns a tuple of tensors (None where an output was not
// wanted), or the status of a failed call as an int.  Unfit tensors raise ValueError.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/core/InferenceMode.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>
#include <cstring>
#include <initializer_list>
#include <optional>
#include <string>

#include "hg.h"

namespace {

struct Api {
  decltype(&hg_rms_norm) rms_norm = nullptr;
  decltype(&hg_rms_norm_grad) rms_norm_grad = nullptr;
  decltype(&hg_rms_norm_grad_workspace) rms_norm_grad_workspace = nullptr;
  decltype(&hg_linear) linear = nullptr;
  decltype(&hg_linear_workspace) linear_workspace = nullptr;
  decltype(&hg_linear_grad) linear_grad = nullptr;
  decltype(&hg_linear_grad_workspace) linear_grad_workspace = nullptr;
  decltype(&hg_distill) distill = nullptr;
  decltype(&hg_layer_norm) layer_norm = nullptr;
  decltype(&hg_layer_norm_grad) layer_norm_grad = nullptr;
  decltype(&hg_layer_norm_grad_workspace) layer_norm_grad_workspace = nullptr;
  decltype(&hg_embed) embed = nullptr;
  decltype(&hg_embed_grad) embed_grad = nullptr;
  decltype(&hg_embed_grad_workspace) embed_grad_workspace = nullptr;
  decltype(&hg_quantize) quantize = nullptr;
  decltype(&hg_dequantize) dequantize = nullptr;
  decltype(&hg_linear_grad_kept) linear_grad_kept = nullptr;
  decltype(&hg_linear_grad_kept_workspace) linear_grad_kept_workspace = nullptr;
} api;
constexpr int kEntries = int(sizeof(Api) / sizeof(void *));

// An argument that does not fit: ValueError.
struct Unfit : std::exception {
  std::string text;
  explicit Unfit(std::string t) : text(std::move(t)) {}
  const char *what() const noexcept override { return text.c_str(); }
};
// A Python error that is set already.
struct PythonError : std::exception {};

std::string shape_text(const at::Tensor &t) {
  std::string s = "(";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + ")";
}

typedef std::initializer_list<at::ScalarType> Types;
const Types kFloats = {at::kFloat, at::kHalf, at::kBFloat16};

int32_t code_of(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return HG_DT_F32;
    case at::kHalf: return HG_DT_F16;
    case at::kBFloat16: return HG_DT_BF16;
    case at::kFloat8_e4m3fn: return HG_DT_E4M3;
    case at::kChar: return HG_DT_I8;
    default: return HG_DT_NONE;
  }
}

const at::Tensor *given(PyObject *o, const char *name) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) throw Unfit(std::string(name) + ": a tensor is wanted");
  return &THPVariable_Unpack(o);
}

// The forward calls record nothing for autograd: a gradient that torch would be asked for later is
// refused here, not dropped.
void no_gradient(std::initializer_list<PyObject *> tensors) {
  if (!c10::GradMode::is_enabled()) return;
  for (PyObject *o : tensors)
    if (o != Py_None && THPVariable_Check(o) && THPVariable_Unpack(o).requires_grad())
      throw Unfit("a tensor requires a gradient, and this call records none: call it under "
                  "torch.no_grad(), or detach the tensor (the backward passes are calls of their own)");
}

void check_type(const at::Tensor &t, const char *name, Types types) {
  for (at::ScalarType s : types)
    if (t.scalar_type() == s) return;
  throw Unfit(std::string(name) + ": unsupported dtype " + at::toString(t.scalar_type()));
}
void check_float(at::ScalarType t, const char *name) {
  if (t != at::kFloat && t != at::kHalf && t != at::kBFloat16)
    throw Unfit(std::string(name) + ": unsupported dtype " + at::toString(t));
}
void check_device(const at::Tensor &t, const char *name, std::optional<at::Device> device) {
  if (!t.device().is_cuda() || (device && t.device() != *device))
    throw Unfit(std::string(name) + ": on " + t.device().str() + ", not on " +
                (device ? device->str() : "a GPU"));
}

// A matrix with contiguous columns (a copy where they are not); rows or cols of -1: any.
at::Tensor matrix(PyObject *o, const char *name, Types types,
                  std::optional<at::Device> device = std::nullopt, int64_t rows = -1,
                  int64_t cols = -1) {
  const at::Tensor *t = given(o, name);
  if (!t || t->dim() != 2) throw Unfit(std::string(name) + ": a 2-D tensor is wanted");
  check_device(*t, name, device);
  check_type(*t, name, types);
  if ((rows >= 0 && t->size(0) != rows) || (cols >= 0 && t->size(1) != cols))
    throw Unfit(std::string(name) + ": shape " + shape_text(*t) + ", not (" +
                (rows < 0 ? "any" : std::to_string(rows)) + ", " +
                (cols < 0 ? "any" : std::to_string(cols)) + ")");
  if (t->size(1) > 1 && t->stride(1) != 1) return t->contiguous();
  return *t;
}
at::Tensor vector(PyObject *o, const char *name, Types types, at::Device device, int64_t n) {
  const at::Tensor *t = given(o, name);
  if (!t || t->dim() != 1 || (n >= 0 && t->size(0) != n))
    throw Unfit(std::string(name) + ": a 1-D tensor" +
                (n >= 0 ? " of " + std::to_string(n) : std::string()) + " is wanted");
  check_device(*t, name, device);
  check_type(*t, name, types);
  return t->is_contiguous() ? *t : t->contiguous();
}
template <typename F>
at::Tensor optional(PyObject *o, F f) {
  return o == Py_None ? at::Tensor() : f(o);
}

void *ptr(const at::Tensor &t) { return t.defined() && t.numel() ? t.data_ptr() : nullptr; }
// Elements between rows (a matrix of one row may report any).
int64_t stride(const at::Tensor &t) {
  return !t.defined() ? 0 : (t.size(0) > 1 ? t.stride(0) : t.size(1));
}

at::Tensor make(at::IntArrayRef shape, at::ScalarType type, at::Device device) {
  return at::empty(shape, at::TensorOptions().dtype(type).device(device));
}
at::Tensor workspace(int64_t bytes, at::Device device) {
  return bytes > 0 ? make({bytes}, at::kByte, device) : at::Tensor();
}
int64_t bytes_of(const at::Tensor &t) { return t.defined() ? t.numel() : 0; }

double number(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PythonError();
  return v;
}
int64_t integer(PyObject *o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PythonError();
  return v;
}
bool truth(PyObject *o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw PythonError();
  return v;
}
at::ScalarType type_or(PyObject *o, at::ScalarType otherwise, const char *name) {
  if (o == Py_None) return otherwise;
  if (!THPDtype_Check(o)) throw Unfit(std::string(name) + ": a torch.dtype is wanted");
  return reinterpret_cast<THPDtype *>(o)->scalar_type;
}

PyObject *result(hg_status st, std::initializer_list<at::Tensor> tensors) {
  if (st != HG_OK) return PyLong_FromLong(st);
  PyObject *t = PyTuple_New(Py_ssize_t(tensors.size()));
  Py_ssize_t i = 0;
  for (const at::Tensor &x : tensors) {
    if (!t) return nullptr;
    PyObject *o = Py_None;
    if (x.defined()) {
      o = THPVariable_Wrap(x);
    } else {
      Py_INCREF(o);
    }
    if (!o) {
      Py_DECREF(t);
      return nullptr;
    }
    PyTuple_SET_ITEM(t, i++, o);
  }
  return t;
}

hipStream_t current_stream(at::Device device) {
  return c10::hip::getCurrentHIPStream(device.index()).stream();
}

// A call's body: C++ exceptions become Python errors.
template <typename F>
PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  if (!api.distill) {
    PyErr_SetString(PyExc_RuntimeError, "bind() has not been called");
    return nullptr;
  }
  try {
    return f();
  } catch (const PythonError &) {
  } catch (const Unfit &e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// x, and the rows that ids (or all of x's) stand for.
struct Taken {
  at::Tensor x, ids;
  int64_t rows;
  Taken(PyObject *px, PyObject *pids) {
    x = matrix(px, "x", kFloats);
    ids = optional(pids, [&](PyObject *o) { return vector(o, "ids", {at::kLong}, x.device(), -1); });
    rows = ids.defined() ? ids.size(0) : x.size(0);
  }
};
at::Tensor norm_weight(PyObject *o, const at::Tensor &x, const char *name = "weight") {
  return optional(o, [&](PyObject *w) {
    return vector(w, name, {at::kFloat, x.scalar_type()}, x.device(), x.size(1));
  });
}
int32_t code_or_none(const at::Tensor &t) {
  return t.defined() ? code_of(t.scalar_type()) : HG_DT_NONE;
}

// rms_norm(x, weight, residual, ids, eps, out_dtype) -> (y, sum, scale)
PyObject *rms_norm(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject * {
    no_gradient({args[0], args[1], args[2]});
    const Taken t(args[0], args[3]);
    const at::Tensor &x = t.x;
    const auto dev = x.device();
    const auto type = x.scalar_type();
    const int64_t rows = t.rows, dim = x.size(1);
    const at::Tensor w = norm_weight(args[1], x);
    const at::Tensor r = optional(args[2], [&](PyObject *o) {
      return matrix(o, "residual", {type}, dev, rows, dim);
    });
    const auto out = type_or(args[5], type, "out_dtype");
    if (out != type && out != at::kFloat8_e4m3fn)
      throw Unfit("out_dtype: neither x's nor torch.float8_e4m3fn");
    const c10::DeviceGuard guard(dev);
    const at::Tensor y = make({rows, dim}, out, dev);
    const at::Tensor sum = r.defined() ? make({rows, dim}, type, dev) : at::Tensor();
    const at::Tensor scale = out != type ? make({rows}, at::kFloat, dev) : at::Tensor();
    hg_norm_args a{};
    a.rows = rows;
    a.dim = dim;
    a.dtype = code_of(type);
    a.out_dtype = code_of(out);
    a.weight_dtype = code_or_none(w);
    a.eps = float(number(args[4]));
    a.x = ptr(x);
    a.x_stride = stride(x);
    a.x_rows = x.size(0);
    a.ids = static_cast<const int64_t *>(ptr(t.ids));
    a.residual = ptr(r);
    a.residual_stride = stride(r);
    a.weight = ptr(w);
    a.y = ptr(y);
    a.y_stride = dim;
    a.scale = static_cast<float *>(ptr(scale));
    a.sum = ptr(sum);
    a.sum_stride = dim;
    return result(api.rms_norm(&a, current_stream(dev)), {y, sum, scale});
  });
}

// rms_norm_grad(dy, x, weight, dsum, ids, eps, want_dx, want_dweight or None) -> (dx, dweight)
PyObject *rms_norm_grad(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject * {
    const Taken t(args[1], args[4]);
    const at::Tensor &x = t.x;
    const auto dev = x.device();
    const auto type = x.scalar_type();
    const int64_t rows = t.rows, dim = x.size(1);
    const at::Tensor dy = matrix(args[0], "dy", {type}, dev, rows, dim);
    const at::Tensor ds = optional(args[3], [&](PyObject *o) {
      return matrix(o, "dsum", {type}, dev, rows, dim);
    });
    const at::Tensor w = norm_weight(args[2], x);
    const bool want_dw = args[7] == Py_None ? w.defined() : truth(args[7]);
    const c10::DeviceGuard guard(dev);
    const at::Tensor dx = truth(args[6]) ? make({rows, dim}, type, dev) : at::Tensor();
    const at::Tensor dw = want_dw ? make({dim}, at::kFloat, dev) : at::Tensor();
    const at::Tensor ws = workspace(want_dw ? api.rms_norm_grad_workspace(rows, dim) : 0, dev);
    hg_norm_grad_args a{};
    a.rows = rows;
    a.dim = dim;
    a.dtype = code_of(type);
    a.weight_dtype = code_or_none(w);
    a.eps = float(number(args[5]));
    a.x = ptr(x);
    a.x_stride = stride(x);
    a.x_rows = x.size(0);
    a.ids = static_cast<const int64_t *>(ptr(t.ids));
    a.weight = ptr(w);
    a.dy = ptr(dy);
    a.dy_stride = stride(dy);
    a.dsum = ptr(ds);
    a.dsum_stride = stride(ds);
    a.dx = ptr(dx);
    a.dx_stride = dim;
    a.dweight = static_cast<float *>(ptr(dw));
    a.workspace = ptr(ws);
    a.workspace_bytes = bytes_of(ws);
    return result(api.rms_norm_grad(&a, current_stream(dev)), {dx, dw});
  });
}

// layer_norm(x, weight, bias, residual, ids, eps, out_dtype) -> (y, sum, scale)
PyObject *layer_norm(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject * {
    no_gradient({args[0], args[1], args[2], args[3]});
    const Taken t(args[0], args[4]);
    const at::Tensor &x = t.x;
    const auto dev = x.device();
    const auto type = x.scalar_type();
    const int64_t rows = t.rows, dim = x.size(1);
    const at::Tensor w = norm_weight(args[1], x), b = norm_weight(args[2], x, "bias");
    const at::Tensor r = optional(args[3], [&](PyObject *o) {
      return matrix(o, "residual", {type}, dev, rows, dim);
    });
    const auto out = type_or(args[6], type, "out_dtype");
    const bool eight = out == at::kFloat8_e4m3fn || out == at::kChar;
    if (out != type && !eight)
      throw Unfit("out_dtype: none of x's, torch.float8_e4m3fn, torch.int8");
    const c10::DeviceGuard guard(dev);
    const at::Tensor y = make({rows, dim}, out, dev);
    const at::Tensor sum = r.defined() ? make({rows, dim}, type, dev) : at::Tensor();
    const at::Tensor scale = eight ? make({rows}, at::kFloat, dev) : at::Tensor();
    hg_layer_norm_args a{};
    a.rows = rows;
    a.dim = dim;
    a.dtype = code_of(type);
    a.out_dtype = code_of(out);
    a.weight_dtype = code_or_none(w);
    a.bias_dtype = code_or_none(b);
    a.eps = float(number(args[5]));
    a.x = ptr(x);
    a.x_stride = stride(x);
    a.x_rows = x.size(0);
    a.ids = static_cast<const int64_t *>(ptr(t.ids));
    a.residual = ptr(r);
    a.residual_stride = stride(r);
    a.weight = ptr(w);
    a.bias = ptr(b);
    a.y = ptr(y);
    a.y_stride = dim;
    a.scale = static_cast<float *>(ptr(scale));
    a.sum = ptr(sum);
    a.sum_stride = dim;
    return result(api.layer_norm(&a, current_stream(dev)), {y, sum, scale});
  });
}

// layer_norm_grad(dy, x, weight, dsum, ids, eps, want_dx, want_dweight or None, want_dbias)
//   -> (dx, dweight, dbias)
PyObject *layer_norm_grad(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject * {
    const Taken t(args[1], args[4]);
    const at::Tensor &x = t.x;
    const auto dev = x.device();
    const auto type = x.scalar_type();
    const int64_t rows = t.rows, dim = x.size(1);
    const at::Tensor dy = matrix(args[0], "dy", {type}, dev, rows, dim);
    const at::Tensor ds = optional(args[3], [&](PyObject *o) {
      return matrix(o, "dsum", {type}, dev, rows, dim);
    });
    const at::Tensor w = norm_weight(args[2], x);
    const bool want_dw = args[7] == Py_None ? w.defined() : truth(args[7]);
    const bool want_db = truth(args[8]);
    const c10::DeviceGuard guard(dev);
    const at::Tensor dx = truth(args[6]) ? make({rows, dim}, type, dev) : at::Tensor();
    const at::Tensor dw = want_dw ? make({dim}, at::kFloat, dev) : at::Tensor();
    const at::Tensor db = want_db ? make({dim}, at::kFloat, dev) : at::Tensor();
    const at::Tensor ws =
        workspace(want_dw || want_db ? api.layer_norm_grad_workspace(rows, dim) : 0, dev);
    hg_layer_norm_grad_args a{};
    a.rows = rows;
    a.dim = dim;
    a.dtype = code_of(type);
    a.weight_dtype = code_or_none(w);
    a.eps = float(number(args[5]));
    a.x = ptr(x);
    a.x_stride = stride(x);
    a.x_rows = x.size(0);
    a.ids = static_cast<const int64_t *>(ptr(t.ids));
    a.weight = ptr(w);
    a.dy = ptr(dy);
    a.dy_stride = stride(dy);
    a.dsum = ptr(ds);
    a.dsum_stride = stride(ds);
    a.dx = ptr(dx);
    a.dx_stride = dim;
    a.dweight = static_cast<float *>(ptr(dw));
    a.dbias = static_cast<float *>(ptr(db));
    a.workspace = ptr(ws);
    a.workspace_bytes = bytes_of(ws);
    return result(api.layer_norm_grad(&a, current_stream(dev)), {dx, dw, db});
  });
}

// embed(table, ids, scale, out_dtype) -> (y,)
PyObject *embed(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(n, 4, [&]() -> PyObject * {
    no_gradient({args[0]});
    const at::Tensor table = matrix(args[0], "table", kFloats);
    const auto dev = table.device();
    const at::Tensor ids = vector(args[1], "ids", {at::kLong}, dev, -1);
    const auto out = type_or(args[3], table.scalar_type(), "out_dtype");
    check_float(out, "out_dtype");
    const int64_t rows = ids.size(0), dim = table.size(1);
    const c10::DeviceGuard guard(dev);
    const at::Tensor y = make({rows, dim}, out, dev);
    hg_embed_args a{};
    a.n = rows;
    a.nodes = table.size(0);
    a.dim = dim;
    a.table_dtype = code_of(table.scalar_type());
    a.out_dtype = code_of(out);
    a.scale = float(number(args[2]));
    a.table = ptr(table);
    a.table_stride = stride(table);
    a.ids = static_cast<const int64_t *>(ptr(ids));
    a.y = ptr(y);
    a.y_stride = dim;
    return result(api.embed(&a, current_stream(dev)), {y});
  });
}

// embed_grad(dy, ids, nodes, scale, out_dtype, into) -> (dtable,)
PyObject *embed_grad(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject * {
    no_gradient({args[5]});  // (written in place)
    const at::Tensor dy = matrix(args[0], "dy", kFloats);
    const auto dev = dy.device();
    const auto type = dy.scalar_type();
    const int64_t rows = dy.size(0), dim = dy.size(1);
    const at::Tensor ids = vector(args[1], "ids", {at::kLong}, dev, rows);
    const int64_t nodes = integer(args[2]);
    const bool add = args[5] != Py_None;
    const auto out = type_or(args[4], at::kFloat, "out_dtype");
    if (out != at::kFloat && (add || out != type))
      throw Unfit(add ? "out_dtype: into is float32" : "out_dtype: neither dy's nor float32");
    if (nodes < 0) throw Unfit("nodes: negative");
    const c10::DeviceGuard guard(dev);
    at::Tensor d;
    if (add) {
      const at::Tensor *const t = given(args[5], "into");
      matrix(args[5], "into", {at::kFloat}, dev, nodes, dim);
      if ((dim > 1 && t->stride(1) != 1) || (nodes > 1 && t->stride(0) < dim))
        throw Unfit("into: its columns are not contiguous, or its rows overlap");
      if (t->is_inference() && !c10::InferenceMode::is_enabled())
        throw Unfit("into: an inference tensor is not written outside of inference mode");
      d = *t;
    } else {
      d = make({nodes, dim}, out, dev);
    }
    const at::Tensor ws =
        workspace(api.embed_grad_workspace(rows, nodes, dim), dev);
    hg_embed_grad_args a{};
    a.n = rows;
    a.nodes = nodes;
    a.dim = dim;
    a.dtype = code_of(type);
    a.out_dtype = code_of(out);
    a.add = add;
    a.scale = float(number(args[3]));
    a.dy = ptr(dy);
    a.dy_stride = stride(dy);
    a.ids = static_cast<const int64_t *>(ptr(ids));
    a.dtable = ptr(d);
    a.dtable_stride = stride(d);
    a.workspace = ptr(ws);
    a.workspace_bytes = bytes_of(ws);
    const hg_status st = api.embed_grad(&a, current_stream(dev));
    // (what autograd has kept of it elsewhere is no longer its value)
    if (add && st == HG_OK && !d.is_inference()) d.unsafeGetTensorImpl()->bump_version();
    return result(st, {d});
  });
}

int32_t group_of(PyObject *o) {
  const int64_t g = integer(o);
  if (g != 0 && g != HG_KEPT_GROUP)
    throw Unfit("group: neither 0 (the row) nor " + std::to_string(HG_KEPT_GROUP));
  return int32_t(g);
}
// The scales of rows x cols integers, contiguous: [rows], or [rows, groups].
at::Tensor scales(PyObject *o, const char *name, int32_t group, at::Device device, int64_t rows,
                  int64_t cols) {
  if (!group) return vector(o, name, {at::kFloat}, device, rows);
  const int64_t groups = (cols + group - 1) / group;
  const at::Tensor t = matrix(o, name, {at::kFloat}, device, rows, groups);
  return t.is_contiguous() ? t : t.contiguous();
}

// quantize(x, group) -> (q, scale)
PyObject *quantize(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(n, 2, [&]() -> PyObject * {
    no_gradient({args[0]});
    const at::Tensor x = matrix(args[0], "x", kFloats);
    const auto dev = x.device();
    const int64_t rows = x.size(0), dim = x.size(1);
    const int32_t group = group_of(args[1]);
    const c10::DeviceGuard guard(dev);
    const at::Tensor q = make({rows, dim}, at::kChar, dev);
    const at::Tensor scale = group ? make({rows, (dim + group - 1) / group}, at::kFloat, dev)
                                   : make({rows}, at::kFloat, dev);
    hg_quantize_args a{};
    a.rows = rows;
    a.dim = dim;
    a.dtype = code_of(x.scalar_type());
    a.group = group;
    a.x = ptr(x);
    a.x_stride = stride(x);
    a.q = static_cast<int8_t *>(ptr(q));
    a.q_stride = dim;
    a.scale = static_cast<float *>(ptr(scale));
    return result(api.quantize(&a, current_stream(dev)), {q, scale});
  });
}

// dequantize(q, scale, group, out_dtype) -> (x,)
PyObject *dequantize(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(n, 4, [&]() -> PyObject * {
    no_gradient({args[1]});
    const at::Tensor q = matrix(args[0], "q", {at::kChar});
    const auto dev = q.device();
    const int64_t rows = q.size(0), dim = q.size(1);
    const int32_t group = group_of(args[2]);
    const at::Tensor scale = scales(args[1], "scale", group, dev, rows, dim);
    const auto out = type_or(args[3], at::kBFloat16, "out_dtype");
    check_float(out, "out_dtype");
    const c10::DeviceGuard guard(dev);
    const at::Tensor x = make({rows, dim}, out, dev);
    hg_dequantize_args a{};
    a.rows = rows;
    a.dim = dim;
    a.dtype = code_of(out);
    a.group = group;
    a.q = static_cast<const int8_t *>(ptr(q));
    a.q_stride = stride(q);
    a.scale = static_cast<const float *>(ptr(scale));
    a.x = ptr(x);
    a.x_stride = dim;
    return result(api.dequantize(&a, current_stream(dev)), {x});
  });
}

// linear(x, w, bias, act, residual, x_scale, w_scale, out_dtype, keep_pre) -> (y, pre)
PyObject *linear(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject * {
    no_gradient({args[0], args[1], args[2], args[4]});
    const at::Tensor x = matrix(args[0], "x", {at::kFloat, at::kHalf, at::kBFloat16,
                                               at::kFloat8_e4m3fn, at::kChar});
    const auto dev = x.device();
    const auto type = x.scalar_type();
    const int64_t m = x.size(0), k = x.size(1);
    const at::Tensor w = matrix(args[1], "w", {type}, dev, -1, k);
    const int64_t nn = w.size(0);
    at::Tensor xs, ws;
    auto out = type;
    if (type == at::kFloat8_e4m3fn || type == at::kChar) {
      out = type_or(args[7], at::kBFloat16, "out_dtype");
      if (args[5] == Py_None || args[6] == Py_None)
        throw Unfit("8-bit operands need x_scale and w_scale");
      xs = vector(args[5], "x_scale", {at::kFloat}, dev, m);
      ws = vector(args[6], "w_scale", {at::kFloat}, dev, nn);
      check_float(out, "out_dtype");
    } else {
      if (args[5] != Py_None || args[6] != Py_None) throw Unfit("scales are for 8-bit operands");
      if (type_or(args[7], type, "out_dtype") != type) throw Unfit("out_dtype: not x's dtype");
    }
    const at::Tensor b = optional(args[2], [&](PyObject *o) {
      return vector(o, "bias", kFloats, dev, nn);
    });
    const at::Tensor r = optional(args[4], [&](PyObject *o) {
      return matrix(o, "residual", {out}, dev, m, nn);
    });
    const c10::DeviceGuard guard(dev);
    const at::Tensor y = make({m, nn}, out, dev);
    const at::Tensor pre = truth(args[8]) ? make({m, nn}, out, dev) : at::Tensor();
    const at::Tensor space = workspace(api.linear_workspace(m, k, nn, code_of(type)), dev);
    hg_linear_args a{};
    a.m = m;
    a.k = k;
    a.n = nn;
    a.dtype = code_of(type);
    a.out_dtype = code_of(out);
    a.bias_dtype = code_or_none(b);
    a.act = int32_t(integer(args[3]));
    a.x = ptr(x);
    a.x_stride = stride(x);
    a.x_scale = static_cast<const float *>(ptr(xs));
    a.w = ptr(w);
    a.w_stride = stride(w);
    a.w_scale = static_cast<const float *>(ptr(ws));
    a.bias = ptr(b);
    a.residual = ptr(r);
    a.residual_stride = stride(r);
    a.y = ptr(y);
    a.y_stride = nn;
    a.pre = ptr(pre);
    a.pre_stride = nn;
    a.workspace = ptr(space);
    a.workspace_bytes = bytes_of(space);
    return result(api.linear(&a, current_stream(dev)), {y, pre});
  });
}

// linear_grad(dy, x, w, pre, act, want_dx, want_dw, want_dbias, dw_dtype, x_scale, pre_scale,
//   group) -> (dx, dw, dbias)
PyObject *linear_grad(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject * {
    const bool kept_x = args[9] != Py_None, kept_pre = args[10] != Py_None;
    const int32_t group = group_of(args[11]);
    at::Tensor x, w, xs, ps;
    if (kept_x) {
      x = matrix(args[1], "x", {at::kChar});
      w = matrix(args[2], "w", kFloats, x.device(), -1, x.size(1));
      xs = scales(args[9], "x_scale", group, x.device(), x.size(0), x.size(1));
    } else {
      x = matrix(args[1], "x", kFloats);
      w = matrix(args[2], "w", {x.scalar_type()}, x.device(), -1, x.size(1));
    }
    const auto dev = x.device();
    const auto type = w.scalar_type();
    const int64_t m = x.size(0), k = x.size(1);
    const int64_t nn = w.size(0);
    const at::Tensor dy = matrix(args[0], "dy", {type}, dev, m, nn);
    const int32_t act = int32_t(integer(args[4]));
    at::Tensor pre;
    if (act != HG_ACT_NONE) {
      if (args[3] == Py_None) throw Unfit("an activation needs pre");
      pre = matrix(args[3], "pre", {kept_pre ? at::kChar : type}, dev, m, nn);
      if (kept_pre) ps = scales(args[10], "pre_scale", group, dev, m, nn);
    } else if (kept_pre) {
      throw Unfit("pre_scale: without an activation there is no pre");
    }
    const auto dw_type = type_or(args[8], type, "dw_dtype");
    if (dw_type != type && dw_type != at::kFloat)
      throw Unfit("dw_dtype: neither w's nor float32");
    const c10::DeviceGuard guard(dev);
    const at::Tensor dx = truth(args[5]) ? make({m, k}, type, dev) : at::Tensor();
    const at::Tensor dw = truth(args[6]) ? make({nn, k}, dw_type, dev) : at::Tensor();
    const at::Tensor db = truth(args[7]) ? make({nn}, at::kFloat, dev) : at::Tensor();
    const bool kept = kept_x || kept_pre;
    const at::Tensor space =
        workspace((kept_x && dw.defined() ? api.linear_grad_kept_workspace
                                          : api.linear_grad_workspace)(m, k, nn, code_of(type), act),
                  dev);
    hg_linear_grad_kept_args all{};
    hg_linear_grad_args &a = all.grad;
    all.group = group;
    all.x_scale = static_cast<const float *>(ptr(xs));
    all.pre_scale = static_cast<const float *>(ptr(ps));
    a.m = m;
    a.k = k;
    a.n = nn;
    a.dtype = code_of(type);
    a.dw_dtype = code_of(dw_type);
    a.act = act;
    a.dy = ptr(dy);
    a.dy_stride = stride(dy);
    a.pre = ptr(pre);
    a.pre_stride = stride(pre);
    a.x = ptr(x);
    a.x_stride = stride(x);
    a.w = ptr(w);
    a.w_stride = stride(w);
    a.dx = ptr(dx);
    a.dx_stride = k;
    a.dw = ptr(dw);
    a.dw_stride = k;
    a.dbias = static_cast<float *>(ptr(db));
    a.workspace = ptr(space);
    a.workspace_bytes = bytes_of(space);
    const auto stream = current_stream(dev);
    return result(kept ? api.linear_grad_kept(&all, stream) : api.linear_grad(&a, stream),
                  {dx, dw, db});
  });
}

// distill(logits, ids, teacher, temperature, row_weight, want_loss, want_grad) -> (loss, grad)
PyObject *distill(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject * {
    // (with the gradient asked for, logits may come from autograd: it goes back by logits.backward(grad))
    if (!truth(args[6])) no_gradient({args[0]});
    const at::Tensor z = matrix(args[0], "logits", kFloats);
    const auto dev = z.device();
    const int64_t rows = z.size(0), classes = z.size(1);
    const at::Tensor ids = matrix(args[1], "ids", {at::kLong}, dev, rows);
    const int64_t top = ids.size(1);
    const at::Tensor t = matrix(args[2], "teacher", kFloats, dev, rows, top);
    const at::Tensor rw = optional(args[4], [&](PyObject *o) {
      return vector(o, "row_weight", {at::kFloat}, dev, rows);
    });
    const c10::DeviceGuard guard(dev);
    const at::Tensor loss = truth(args[5]) ? make({rows}, at::kFloat, dev) : at::Tensor();
    const at::Tensor grad =
        truth(args[6]) ? make({rows, classes}, z.scalar_type(), dev) : at::Tensor();
    hg_distill_args a{};
    a.rows = rows;
    a.classes = classes;
    a.top = int32_t(top > INT32_MAX ? INT32_MAX : top);
    a.dtype = code_of(z.scalar_type());
    a.teacher_dtype = code_of(t.scalar_type());
    a.temperature = float(number(args[3]));
    a.logits = ptr(z);
    a.logits_stride = stride(z);
    a.ids = static_cast<const int64_t *>(ptr(ids));
    a.ids_stride = stride(ids);
    a.teacher = ptr(t);
    a.teacher_stride = stride(t);
    a.row_weight = static_cast<const float *>(ptr(rw));
    a.loss = static_cast<float *>(ptr(loss));
    a.grad = ptr(grad);
    a.grad_stride = classes;
    return result(api.distill(&a, current_stream(dev)), {loss, grad});
  });
}

// bind(addresses of the entry points, in Api's order)
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != kEntries) {
    PyErr_Format(PyExc_TypeError, "bind() takes %d addresses", kEntries);
    return nullptr;
  }
  void *v[kEntries];
  for (int i = 0; i < kEntries; ++i) {
    v[i] = PyLong_AsVoidPtr(args[i]);
    if (!v[i] && PyErr_Occurred()) return nullptr;
  }
  static_assert(sizeof(v) == sizeof(api));
  std::memcpy(static_cast<void *>(&api), v, sizeof(v));
  Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
PyMethodDef method(const char *name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL,
          nullptr};
}

PyMethodDef methods[] = {method<bind>("bind"),
                         method<rms_norm>("rms_norm"),
                         method<rms_norm_grad>("rms_norm_grad"),
                         method<layer_norm>("layer_norm"),
                         method<layer_norm_grad>("layer_norm_grad"),
                         method<embed>("embed"),
                         method<embed_grad>("embed_grad"),
                         method<quantize>("quantize"),
                         method<dequantize>("dequantize"),
                         method<linear>("linear"),
                         method<linear_grad>("linear_grad"),
                         method<distill>("distill"),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_hgdense", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__hgdense(void) { return PyModule_Create(&module); }
