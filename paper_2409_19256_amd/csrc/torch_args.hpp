// What the native modules of the rollout operators share: torch tensors looked over and taken as arguments.  For one source file a module.
#pragma once
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/forward_grad.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "hfreshard.h"

namespace {

using at::Tensor;

PyObject *g_error = nullptr; // HfError(code, name of the call)

struct Wrong {
  const char *name, *what;
};

// the tensor of an argument, null for None; throws Wrong
[[maybe_unused]] const Tensor *given(PyObject *o, const char *name) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) throw Wrong{name, "a tensor is wanted"};
  return &THPVariable_Unpack(o);
}
[[maybe_unused]] const Tensor &wanted(PyObject *o, const char *name) {
  const Tensor *t = given(o, name);
  if (!t) throw Wrong{name, "a tensor is wanted"};
  return *t;
}

// address of a contiguous tensor of a type and shape on the GPU `device`; null for none
template <size_t kN> void *whole(const Tensor *t, const char *name, at::ScalarType type, const int64_t (&shape)[kN], int device) {
  if (!t) return nullptr;
  if (!t->is_cuda() || t->get_device() != device) throw Wrong{name, "a tensor on the operands' GPU is wanted"};
  if (t->scalar_type() != type) throw Wrong{name, "a tensor of another type is wanted"};
  if (t->sizes() != at::IntArrayRef(shape, kN)) throw Wrong{name, "a tensor of another shape is wanted"};
  if (!t->is_contiguous()) throw Wrong{name, "a contiguous tensor is wanted"};
  return t->data_ptr();
}

struct Rows {
  void *at;
  int64_t stride, head_stride;
};
// a tensor of three dimensions whose last one is contiguous
[[maybe_unused]] Rows rows_of(const Tensor &t, const char *name, at::ScalarType type, int64_t a, int64_t b, int64_t c, int device) {
  if (!t.is_cuda() || t.get_device() != device) throw Wrong{name, "a tensor on the operands' GPU is wanted"};
  if (t.scalar_type() != type) throw Wrong{name, "a tensor of another type is wanted"};
  const auto size = t.sizes();
  if (size.size() != 3 || size[0] != a || size[1] != b || size[2] != c) throw Wrong{name, "a tensor of another shape is wanted"};
  const auto stride = t.strides();
  if (stride[2] != 1 && c != 1) throw Wrong{name, "the last dimension has to be contiguous"};
  return {t.data_ptr(), stride[0], stride[1]};
}

[[maybe_unused]] int32_t int32_of(int64_t n, const char *name) {
  if (n > INT32_MAX || n < INT32_MIN) throw Wrong{name, "too large"};
  return (int32_t)n;
}
[[maybe_unused]] int64_t number(PyObject *o) {
  const long long n = PyLong_AsLongLong(o);
  if (n == -1 && PyErr_Occurred()) throw python_error();
  return n;
}
[[maybe_unused]] double real(PyObject *o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1 && PyErr_Occurred()) throw python_error();
  return x;
}
[[maybe_unused]] int32_t bound(PyObject *o, int64_t otherwise, const char *name) { return int32_of(o == Py_None ? otherwise : number(o), name); }

[[maybe_unused]] const hf_kv_cache *cache_of(PyObject *o) {
  if (!PyBytes_Check(o) || PyBytes_GET_SIZE(o) != (Py_ssize_t)sizeof(hf_kv_cache)) throw Wrong{"cache", "an hf_kv_cache in bytes is wanted"};
  return reinterpret_cast<const hf_kv_cache *>(PyBytes_AS_STRING(o));
}
// the buffers of a cache, which have to be where the operands are
[[maybe_unused]] void same_gpu(PyObject *keys, PyObject *values, int device) {
  for (PyObject *o : {keys, values})
    if (const Tensor &t = wanted(o, "cache"); !t.is_cuda() || t.get_device() != device) throw Wrong{"cache", "a cache on the operands' GPU is wanted"};
}
// What torch would take a gradient by: backward, and forward mode, whose tangents live as long as its level and which no_grad does not end.
struct Modes {
  bool backward = c10::GradMode::is_enabled(), forward = torch::autograd::ForwardADLevel::try_get_by_idx(0) != nullptr;
};
// Some operators have no gradient: where torch would take one they refuse, rather than lose it in silence.
[[maybe_unused]] void without_gradient(std::initializer_list<std::pair<const char *, const Tensor *>> tensors, const Modes &modes = Modes()) {
  if (!modes.backward && !modes.forward) return;
  for (const auto &[name, t] : tensors) {
    if (!t) continue;
    if (modes.backward && t->requires_grad()) throw Wrong{name, "no gradient is taken here: detach it, or call under torch.no_grad()"};
    if (modes.forward && t->_fw_grad(0).defined()) throw Wrong{name, "no forward-mode gradient is taken here: unpack the dual tensor"};
  }
}
// what a call has written to, for whoever saved it for a backward pass
[[maybe_unused]] void written(std::initializer_list<const Tensor *> tensors) {
  for (const Tensor *t : tensors)
    if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}
[[maybe_unused]] at::ScalarType type_of(const hf_kv_cache &c) { return c.dtype == HF_BF16 ? at::kBFloat16 : at::kHalf; }
[[maybe_unused]] void *stream_of(PyObject *o) {
  void *s = PyLong_AsVoidPtr(o);
  if (!s && PyErr_Occurred()) throw python_error();
  return s;
}

// what HfError says; always null
[[maybe_unused]] PyObject *failed(int code, const char *call) {
  PyObject *e = PyObject_CallFunction(g_error, "is", code, call);
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  return nullptr;
}
[[maybe_unused]] PyObject *wrap(Tensor t) { return THPVariable_Wrap(std::move(t)); }
[[maybe_unused]] PyObject *again(PyObject *o) {
  Py_INCREF(o);
  return o;
}

template <typename F> PyObject *guarded(Py_ssize_t n, Py_ssize_t want, const F &f) {
  HANDLE_TH_ERRORS
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments are wanted", want);
    return nullptr;
  }
  try {
    return f();
  } catch (const Wrong &w) {
    PyErr_Format(PyExc_ValueError, "%s: %s", w.name, w.what);
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

[[maybe_unused]] hf_logits logits_of(const Tensor &logits, const Tensor *targets, double temperature) {
  if (!logits.is_cuda() || logits.dim() != 2) throw Wrong{"logits", "[rows, vocab] on the GPU is wanted"};
  hf_logits a = {};
  switch (logits.scalar_type()) {
  case at::kBFloat16: a.dtype = HF_BF16; break;
  case at::kHalf: a.dtype = HF_F16; break;
  case at::kFloat: a.dtype = HF_F32; break;
  default: throw Wrong{"logits", "bfloat16, float16 or float32 is wanted"};
  }
  if (logits.stride(1) != 1 && logits.size(1) != 1) throw Wrong{"logits", "the last dimension has to be contiguous"};
  a.logits = logits.data_ptr();
  a.rows = logits.size(0), a.row_stride = logits.stride(0), a.vocab = int32_of(logits.size(1), "logits");
  a.target_bytes = 8;
  if (targets) {
    const bool narrow = targets->scalar_type() == at::kInt;
    a.targets = whole(targets, "targets", narrow ? at::kInt : at::kLong, {a.rows}, logits.get_device());
    a.target_bytes = narrow ? 4 : 8;
  }
  if (!(temperature > 0)) throw Wrong{"temperature", "it has to be positive"};
  a.inv_temperature = (float)(1 / temperature);
  return a;
}

[[maybe_unused]] PyObject *set_error(PyObject *, PyObject *type) {
  Py_XDECREF(g_error);
  g_error = again(type);
  Py_RETURN_NONE;
}

// the references given, all of them or none, as a tuple
[[maybe_unused]] PyObject *tuple_of(std::initializer_list<PyObject *> all) {
  PyObject *t = PyTuple_New((Py_ssize_t)all.size());
  Py_ssize_t i = 0;
  bool whole = t != nullptr;
  for (PyObject *o : all) {
    if (t) PyTuple_SET_ITEM(t, i++, o);
    else Py_XDECREF(o);
    whole = whole && o;
  }
  if (!whole) Py_CLEAR(t);
  return t;
}

template <typename F> PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

} // namespace
