// Python module _rollout: the rollout operators' C calls with torch tensors as arguments.  It looks tensors over, makes the outputs that were not
// given, makes their GPU the current one, and fills the argument structs; the smallest calls wait for the host, and in Python this took two to three times as long as the launch (one step
// of the tiny decoder's attention 15.8 us a call in Python).  rollout.py documents the functions and is what callers import.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/Exceptions.h>
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
const Tensor *given(PyObject *o, const char *name) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) throw Wrong{name, "a tensor is wanted"};
  return &THPVariable_Unpack(o);
}
const Tensor &wanted(PyObject *o, const char *name) {
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
Rows rows_of(const Tensor &t, const char *name, at::ScalarType type, int64_t a, int64_t b, int64_t c, int device) {
  if (!t.is_cuda() || t.get_device() != device) throw Wrong{name, "a tensor on the operands' GPU is wanted"};
  if (t.scalar_type() != type) throw Wrong{name, "a tensor of another type is wanted"};
  const auto size = t.sizes();
  if (size.size() != 3 || size[0] != a || size[1] != b || size[2] != c) throw Wrong{name, "a tensor of another shape is wanted"};
  const auto stride = t.strides();
  if (stride[2] != 1 && c != 1) throw Wrong{name, "the last dimension has to be contiguous"};
  return {t.data_ptr(), stride[0], stride[1]};
}

int32_t int32_of(int64_t n, const char *name) {
  if (n > INT32_MAX || n < INT32_MIN) throw Wrong{name, "too large"};
  return (int32_t)n;
}
int64_t number(PyObject *o) {
  const long long n = PyLong_AsLongLong(o);
  if (n == -1 && PyErr_Occurred()) throw python_error();
  return n;
}
double real(PyObject *o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1 && PyErr_Occurred()) throw python_error();
  return x;
}
int32_t bound(PyObject *o, int64_t otherwise, const char *name) { return int32_of(o == Py_None ? otherwise : number(o), name); }

const hf_kv_cache *cache_of(PyObject *o) {
  if (!PyBytes_Check(o) || PyBytes_GET_SIZE(o) != (Py_ssize_t)sizeof(hf_kv_cache)) throw Wrong{"cache", "an hf_kv_cache in bytes is wanted"};
  return reinterpret_cast<const hf_kv_cache *>(PyBytes_AS_STRING(o));
}
// the buffers of a cache, which have to be where the operands are
void same_gpu(PyObject *keys, PyObject *values, int device) {
  for (PyObject *o : {keys, values})
    if (const Tensor &t = wanted(o, "cache"); !t.is_cuda() || t.get_device() != device) throw Wrong{"cache", "a cache on the operands' GPU is wanted"};
}
// The cache's operators have no backward: where torch would take a gradient they refuse, rather than lose it in silence.
void without_gradient(std::initializer_list<std::pair<const char *, const Tensor *>> tensors) {
  if (!c10::GradMode::is_enabled()) return;
  for (const auto &[name, t] : tensors)
    if (t && t->requires_grad()) throw Wrong{name, "no gradient is taken here: detach it, or call under torch.no_grad()"};
}
// what a call has written to, for whoever saved it for a backward pass
void written(std::initializer_list<const Tensor *> tensors) {
  for (const Tensor *t : tensors)
    if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}
at::ScalarType type_of(const hf_kv_cache &c) { return c.dtype == HF_BF16 ? at::kBFloat16 : at::kHalf; }
void *stream_of(PyObject *o) {
  void *s = PyLong_AsVoidPtr(o);
  if (!s && PyErr_Occurred()) throw python_error();
  return s;
}

// what HfError says; always null
PyObject *failed(int code, const char *call) {
  PyObject *e = PyObject_CallFunction(g_error, "is", code, call);
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  return nullptr;
}
PyObject *wrap(Tensor t) { return THPVariable_Wrap(std::move(t)); }
PyObject *again(PyObject *o) {
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

// (cache, its keys, its values, stream, k, v, slots, positions, cos, sin, q, q_out, interleaved) -> q_out
PyObject *append(PyObject *, PyObject *const *arg, Py_ssize_t n_args) {
  return guarded(n_args, 13, [&]() -> PyObject * {
    const hf_kv_cache &c = *cache_of(arg[0]);
    const Tensor &k = wanted(arg[4], "k"), &v = wanted(arg[5], "v"), &slots = wanted(arg[6], "slots");
    const Tensor *positions = given(arg[7], "positions"), *cos = given(arg[8], "cos"), *sin = given(arg[9], "sin"), *q = given(arg[10], "q");
    const at::ScalarType type = type_of(c);
    if (!k.is_cuda() || k.dim() != 3) throw Wrong{"k", "[token, KV head, element] on the GPU is wanted"};
    const int device = k.get_device();
    same_gpu(arg[1], arg[2], device);
    const c10::DeviceGuard current(k.device());
    const int64_t n = k.size(0);
    hf_append a = {};
    const Rows ks = rows_of(k, "k", type, n, c.n_kv_heads, c.head_dim, device), vs = rows_of(v, "v", type, n, c.n_kv_heads, c.head_dim, device);
    a.k = ks.at, a.k_stride = ks.stride, a.k_head_stride = ks.head_stride;
    a.v = vs.at, a.v_stride = vs.stride, a.v_head_stride = vs.head_stride;
    a.n_tokens = int32_of(n, "k");
    a.slots = static_cast<const int64_t *>(whole(&slots, "slots", at::kLong, {n}, device));
    if (cos) {
      if (cos->dim() != 2 || !sin || !positions) throw Wrong{"cos", "[position, pair] with sin and positions is wanted"};
      const int64_t table = cos->size(0), pairs = cos->size(1);
      a.cos = static_cast<const float *>(whole(cos, "cos", at::kFloat, {table, pairs}, device));
      a.sin = static_cast<const float *>(whole(sin, "sin", at::kFloat, {table, pairs}, device));
      a.positions = static_cast<const int32_t *>(whole(positions, "positions", at::kInt, {n}, device));
      a.rot_dim = int32_of(2 * pairs, "cos"), a.n_positions = int32_of(table, "cos");
    }
    const Tensor *out = q ? given(arg[11], "q_out") : nullptr;
    without_gradient({{"cache", &wanted(arg[1], "cache")}, {"cache", &wanted(arg[2], "cache")}, {"k", &k}, {"v", &v}, {"q", q}, {"q_out", out}});
    PyObject *result = nullptr;
    Tensor made;
    if (q) {
      if (q->dim() != 3) throw Wrong{"q", "[token, query head, element] is wanted"};
      const int64_t heads = q->size(1);
      const Rows qs = rows_of(*q, "q", type, n, heads, c.head_dim, device);
      a.q = qs.at, a.q_stride = qs.stride, a.q_head_stride = qs.head_stride, a.n_q_heads = int32_of(heads, "q");
      if (!out) made = at::empty({n, heads, c.head_dim}, q->options());
      const Rows os = rows_of(out ? *out : made, "q_out", type, n, heads, c.head_dim, device);
      a.q_out = os.at, a.q_out_stride = os.stride, a.q_out_head_stride = os.head_stride;
      if (out) result = arg[11];
    }
    const int interleaved = PyObject_IsTrue(arg[12]);
    if (interleaved < 0) throw python_error();
    a.flags = interleaved ? HF_ROT_INTERLEAVED : 0;
    if (const int code = hf_append_kv(&c, &a, stream_of(arg[3]))) return failed(code, "hf_append_kv");
    written({&wanted(arg[1], "cache"), &wanted(arg[2], "cache"), out});
    return made.defined() ? wrap(std::move(made)) : again(result ? result : Py_None);
  });
}

// (cache, its keys, its values, stream, q, suffix_lens, suffix_pages, group_offsets, prefix_lens, prefix_pages, max_group, max_prefix, max_suffix, scale, out, lse, workspace)
// -> (out, lse)
PyObject *attend(PyObject *, PyObject *const *arg, Py_ssize_t n_args) {
  return guarded(n_args, 17, [&]() -> PyObject * {
    const hf_kv_cache &c = *cache_of(arg[0]);
    const Tensor &q = wanted(arg[4], "q"), &lens = wanted(arg[5], "suffix_lens"), &pages = wanted(arg[6], "suffix_pages");
    const Tensor *offsets = given(arg[7], "group_offsets"), *prefix_lens = given(arg[8], "prefix_lens"), *prefix_pages = given(arg[9], "prefix_pages");
    const Tensor *out = given(arg[14], "out"), *lse = given(arg[15], "lse"), *workspace = given(arg[16], "workspace");
    const at::ScalarType type = type_of(c);
    if (!q.is_cuda() || q.dim() != 3) throw Wrong{"q", "[sequence, query head, element] on the GPU is wanted"};
    const int device = q.get_device();
    same_gpu(arg[1], arg[2], device);
    const c10::DeviceGuard current(q.device());
    without_gradient({{"cache", &wanted(arg[1], "cache")}, {"cache", &wanted(arg[2], "cache")}, {"q", &q}, {"out", out}, {"lse", lse}});
    const int64_t n = q.size(0), heads = q.size(1);
    hf_attention a = {};
    const Rows qs = rows_of(q, "q", type, n, heads, c.head_dim, device);
    a.q = qs.at, a.q_stride = qs.stride, a.q_head_stride = qs.head_stride;
    a.n_seqs = int32_of(n, "q"), a.n_q_heads = int32_of(heads, "q");
    Tensor made_out, made_lse, made_workspace;
    if (!out) made_out = at::empty({n, heads, c.head_dim}, q.options());
    const Rows os = rows_of(out ? *out : made_out, "out", type, n, heads, c.head_dim, device);
    a.out = os.at, a.out_stride = os.stride, a.out_head_stride = os.head_stride;
    if (!lse) made_lse = at::empty({n, heads}, q.options().dtype(at::kFloat));
    a.lse = static_cast<float *>(whole(lse ? lse : &made_lse, "lse", at::kFloat, {n, heads}, device));
    if (pages.dim() != 2) throw Wrong{"suffix_pages", "[sequence, page] is wanted"};
    const int64_t width = pages.size(1);
    a.suffix_lens = static_cast<const int32_t *>(whole(&lens, "suffix_lens", at::kInt, {n}, device));
    a.suffix_pages = static_cast<const int32_t *>(whole(&pages, "suffix_pages", at::kInt, {n, width}, device));
    a.suffix_width = int32_of(width, "suffix_pages");
    int64_t prefix_width = 0;
    if (offsets) {
      if (!prefix_lens || !prefix_pages || prefix_pages->dim() != 2) throw Wrong{"prefix_pages", "[prompt, page] and prefix_lens are wanted"};
      const int64_t groups = prefix_pages->size(0);
      prefix_width = prefix_pages->size(1);
      a.group_offsets = static_cast<const int32_t *>(whole(offsets, "group_offsets", at::kInt, {groups + 1}, device));
      a.prefix_lens = static_cast<const int32_t *>(whole(prefix_lens, "prefix_lens", at::kInt, {groups}, device));
      a.prefix_pages = static_cast<const int32_t *>(whole(prefix_pages, "prefix_pages", at::kInt, {groups, prefix_width}, device));
      a.n_groups = int32_of(groups, "prefix_pages"), a.prefix_width = int32_of(prefix_width, "prefix_pages");
    }
    a.max_group = bound(arg[10], n, "max_group");
    a.max_prefix = bound(arg[11], std::min<int64_t>(prefix_width * c.page_tokens, INT32_MAX), "max_prefix");
    a.max_suffix = bound(arg[12], std::min<int64_t>(width * c.page_tokens, INT32_MAX), "max_suffix");
    a.scale = arg[13] == Py_None ? (float)(1 / std::sqrt((double)c.head_dim)) : (float)real(arg[13]);
    if (workspace) {
      if (!workspace->is_cuda() || workspace->get_device() != device || !workspace->is_contiguous()) throw Wrong{"workspace", "a contiguous tensor on the operands' GPU is wanted"};
      a.workspace = workspace->data_ptr(), a.workspace_bytes = workspace->nbytes();
    } else {
      const size_t size = hf_attend_workspace_bytes(&c, &a);
      if (size == (size_t)-1) return failed(HF_EINVAL, "hf_attend_workspace_bytes");
      if (size) {
        made_workspace = at::empty({(int64_t)size}, q.options().dtype(at::kByte));
        a.workspace = made_workspace.data_ptr(), a.workspace_bytes = size;
      }
    }
    if (const int code = hf_attend(&c, &a, stream_of(arg[3]))) return failed(code, "hf_attend");
    written({out, lse, workspace});
    PyObject *first = out ? again(arg[14]) : wrap(std::move(made_out)), *second = lse ? again(arg[15]) : wrap(std::move(made_lse));
    PyObject *both = first && second ? PyTuple_Pack(2, first, second) : nullptr;
    Py_XDECREF(first);
    Py_XDECREF(second);
    return both;
  });
}

hf_logits logits_of(const Tensor &logits, const Tensor *targets, PyObject *temperature) {
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
  const double t = real(temperature);
  if (!(t > 0)) throw Wrong{"temperature", "it has to be positive"};
  a.inv_temperature = (float)(1 / t);
  return a;
}

// (stream, logits, targets, temperature, top, apart) -> (logprob, entropy, lse and norm in one, ids, log probabilities, logprob in a tensor of its own if it is wanted apart)
PyObject *token_logprobs(PyObject *, PyObject *const *arg, Py_ssize_t n_args) {
  return guarded(n_args, 6, [&]() -> PyObject * {
    const Tensor &logits = wanted(arg[1], "logits"), *targets = given(arg[2], "targets");
    const hf_logits a = logits_of(logits, targets, arg[3]);
    const c10::DeviceGuard current(logits.device());
    const int64_t top = number(arg[4]);
    if (top < 0 || top > HF_MAX_TOP) throw Wrong{"top", "0 to HF_MAX_TOP is wanted"};
    const auto options = logits.options().dtype(at::kFloat);
    Tensor stats = at::empty({5 * a.rows}, options), ids, values, logprob;
    float *s = static_cast<float *>(stats.data_ptr());
    hf_logprobs o = {};
    o.logprob = targets ? s : nullptr, o.entropy = s + a.rows, o.lse = s + 2 * a.rows, o.norm = s + 3 * a.rows, o.top_n = (int32_t)top;
    if (top) {
      ids = at::empty({a.rows, top}, options.dtype(at::kInt));
      values = at::empty({a.rows, top}, options);
      o.top_ids = static_cast<int32_t *>(ids.data_ptr()), o.top_logprobs = static_cast<float *>(values.data_ptr());
    }
    if (targets && arg[5] == Py_True) {
      logprob = at::empty({a.rows}, options);
      o.logprob = static_cast<float *>(logprob.data_ptr());
    }
    if (const int code = hf_token_logprobs(&a, &o, stream_of(arg[0]))) return failed(code, "hf_token_logprobs");
    const auto made = [](Tensor &t) { return t.defined() ? wrap(std::move(t)) : again(Py_None); };
    PyObject *x = made(stats), *y = made(ids), *z = made(values), *w = made(logprob);
    PyObject *all = x && y && z && w ? PyTuple_Pack(4, x, y, z, w) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    Py_XDECREF(z);
    Py_XDECREF(w);
    return all;
  });
}

// (stream, logits, targets, norm, entropy, grad_logprob, grad_entropy, temperature, out) -> out
PyObject *token_logprobs_back(PyObject *, PyObject *const *arg, Py_ssize_t n_args) {
  return guarded(n_args, 9, [&]() -> PyObject * {
    const Tensor &logits = wanted(arg[1], "logits"), &targets = wanted(arg[2], "targets"), &norm = wanted(arg[3], "norm");
    const hf_logits a = logits_of(logits, &targets, arg[7]);
    const c10::DeviceGuard current(logits.device());
    const int device = logits.get_device();
    hf_logprobs_grad g = {};
    g.norm = static_cast<const float *>(whole(&norm, "norm", at::kFloat, {a.rows, 2}, device));
    g.entropy = static_cast<const float *>(whole(given(arg[4], "entropy"), "entropy", at::kFloat, {a.rows}, device));
    g.grad_logprob = static_cast<const float *>(whole(given(arg[5], "grad_logprob"), "grad_logprob", at::kFloat, {a.rows}, device));
    g.grad_entropy = static_cast<const float *>(whole(given(arg[6], "grad_entropy"), "grad_entropy", at::kFloat, {a.rows}, device));
    const Tensor *out = given(arg[8], "out");
    Tensor made;
    if (!out) made = at::empty(logits.sizes(), logits.options());
    const Tensor &to = out ? *out : made;
    if (!to.is_cuda() || to.get_device() != device || to.scalar_type() != logits.scalar_type() || to.sizes() != logits.sizes()) throw Wrong{"out", "a tensor like the logits is wanted"};
    if (to.stride(1) != 1 && to.size(1) != 1) throw Wrong{"out", "the last dimension has to be contiguous"};
    g.dlogits = to.data_ptr(), g.dlogits_stride = to.stride(0);
    if (const int code = hf_token_logprobs_back(&a, &g, stream_of(arg[0]))) return failed(code, "hf_token_logprobs_back");
    written({out});
    return out ? again(arg[8]) : wrap(std::move(made));
  });
}

PyObject *set_error(PyObject *, PyObject *type) {
  Py_XDECREF(g_error);
  g_error = again(type);
  Py_RETURN_NONE;
}

template <typename F> PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }
PyMethodDef g_methods[] = {{"append", fast(append), METH_FASTCALL, nullptr},
                           {"attend", fast(attend), METH_FASTCALL, nullptr},
                           {"token_logprobs", fast(token_logprobs), METH_FASTCALL, nullptr},
                           {"token_logprobs_back", fast(token_logprobs_back), METH_FASTCALL, nullptr},
                           {"set_error", set_error, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_rollout", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__rollout(void) { return PyModule_Create(&g_module); }
