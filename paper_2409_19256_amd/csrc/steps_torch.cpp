// Python module _steps: the C calls of what surrounds a rollout's steps, with torch tensors as arguments, as _rollout makes those of the others.
// rollout.py documents the functions and is what callers import.
#include "torch_args.hpp"

namespace {

// a tensor [rows, n] of one of two types on the GPU whose last dimension is contiguous
struct Matrix {
  const void *at;
  int64_t stride;
};
Matrix matrix_of(const Tensor &t, const char *name, int64_t rows, int64_t n, int device) {
  if (!t.is_cuda() || t.get_device() != device) throw Wrong{name, "a tensor on the operands' GPU is wanted"};
  if (t.dim() != 2 || t.size(0) != rows || (n >= 0 && t.size(1) != n)) throw Wrong{name, "a tensor of another shape is wanted"};
  if (t.stride(1) != 1 && t.size(1) > 1) throw Wrong{name, "the last dimension has to be contiguous"};
  return {t.data_ptr(), t.stride(0)};
}
const float *per_row(PyObject *o, const char *name, int64_t rows, int device) { return static_cast<const float *>(whole(given(o, name), name, at::kFloat, {rows}, device)); }
void *like(const Tensor &t, const Tensor &logits) {
  if (!t.is_cuda() || t.get_device() != logits.get_device() || t.scalar_type() != logits.scalar_type() || t.sizes() != logits.sizes()) throw Wrong{"out", "a tensor like the logits is wanted"};
  if (t.stride(1) != 1 && t.size(1) != 1) throw Wrong{"out", "the last dimension has to be contiguous"};
  return t.data_ptr();
}

// The outputs of a call that its caller did not give, and a small workspace, in one allocation: the smallest calls wait for the host, which takes 0.65 us to allocate a tensor
// (room for a token in 256 rows 7.3 -> 4.9 us a call).
class Made {
  static constexpr int64_t kSmall = 1 << 16; // a larger workspace does not stay with the outputs
  struct One {
    const char *name;
    Tensor tensor;
    at::ScalarType type;
    c10::SmallVector<int64_t, 4> shape;
    int64_t at;
    void **to;
  };
  c10::SmallVector<One, 8> all_;
  const Tensor &beside_;
  int64_t size_ = 0;
  Tensor store_, workspace_;
  int64_t take(int64_t bytes) {
    const int64_t at = size_;
    size_ += (bytes + 15) / 16 * 16;
    return at;
  }

public:
  explicit Made(const Tensor &beside) : beside_(beside) {}
  // `to` points to what the caller gave now, or to a new tensor of this type and shape after make(); returns the number of a new one, else -1
  template <typename T> int output(PyObject *o, const char *name, at::ScalarType type, at::IntArrayRef shape, T **to) {
    if (const Tensor *t = given(o, name)) {
      if (!t->is_cuda() || t->get_device() != beside_.get_device()) throw Wrong{name, "a tensor on the operands' GPU is wanted"};
      if (t->scalar_type() != type || t->sizes() != shape || !t->is_contiguous()) throw Wrong{name, "a contiguous tensor of the output's type and shape is wanted"};
      *to = static_cast<T *>(t->data_ptr());
      return -1;
    }
    int64_t n = c10::elementSize(type);
    for (const int64_t d : shape) n *= d;
    all_.push_back({name, Tensor(), type, {shape.begin(), shape.end()}, take(n), reinterpret_cast<void **>(to)});
    return (int)all_.size() - 1;
  }
  // and the workspace: the caller's, or a new one of `bytes`
  template <typename A> void make(A &a, size_t bytes, PyObject *workspace) {
    int64_t at = -1;
    if (const Tensor *t = given(workspace, "workspace")) {
      if (!t->is_cuda() || t->get_device() != beside_.get_device() || !t->is_contiguous()) throw Wrong{"workspace", "a contiguous tensor on the operands' GPU is wanted"};
      a.workspace = t->data_ptr(), a.workspace_bytes = t->nbytes();
    } else if ((int64_t)bytes <= kSmall) {
      at = take((int64_t)bytes), a.workspace_bytes = bytes;
    } else {
      workspace_ = at::empty({(int64_t)bytes}, beside_.options().dtype(at::kByte));
      a.workspace = workspace_.data_ptr(), a.workspace_bytes = bytes;
    }
    make();
    if (at >= 0) a.workspace = static_cast<char *>(store_.data_ptr()) + at;
  }
  void make() {
    if (all_.size() == 0 && size_ == 0) return;
    store_ = at::empty({size_ ? size_ : 16}, beside_.options().dtype(at::kByte));
    char *base = static_cast<char *>(store_.data_ptr());
    for (One &o : all_) {
      o.tensor = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(store_.storage()), store_.key_set(), c10::scalarTypeToTypeMeta(o.type));
      o.tensor.unsafeGetTensorImpl()->set_storage_offset(o.at / (int64_t)c10::elementSize(o.type));
      o.tensor.unsafeGetTensorImpl()->set_sizes_contiguous(o.shape);
      *o.to = base + o.at;
    }
  }
  PyObject *result(int made, PyObject *o) { return made >= 0 ? wrap(std::move(all_[made].tensor)) : again(o); }
};

// (stream, logits, tokens, lens, prompt_lens, repetition, frequency, presence, bias_ids, bias, allowed, allowed_rows, out) -> out
PyObject *adjust(PyObject *, PyObject *const *arg, Py_ssize_t n_args) {
  return guarded(n_args, 13, [&]() -> PyObject * {
    const Tensor &logits = wanted(arg[1], "logits"), *tokens = given(arg[2], "tokens"), *bias_ids = given(arg[8], "bias_ids"), *bias = given(arg[9], "bias");
    const Tensor *allowed = given(arg[10], "allowed"), *allowed_rows = given(arg[11], "allowed_rows"), *out = given(arg[12], "out");
    const hf_logits x = logits_of(logits, nullptr, 1.);
    const int device = logits.get_device();
    const c10::DeviceGuard current(logits.device());
    without_gradient({{"logits", &logits}, {"repetition", given(arg[5], "repetition")}, {"frequency", given(arg[6], "frequency")}, {"presence", given(arg[7], "presence")}, {"bias", bias}, {"out", out}});
    hf_adjustment a = {};
    a.logits = x.logits, a.rows = x.rows, a.row_stride = x.row_stride, a.dtype = x.dtype, a.vocab = x.vocab;
    if (tokens) {
      const bool narrow = tokens->scalar_type() == at::kInt;
      if (!narrow && tokens->scalar_type() != at::kLong) throw Wrong{"tokens", "int32 or int64 is wanted"};
      const Matrix m = matrix_of(*tokens, "tokens", a.rows, -1, device);
      a.tokens = m.at, a.tokens_stride = m.stride, a.token_bytes = narrow ? 4 : 8, a.width = int32_of(tokens->size(1), "tokens");
      a.lens = static_cast<const int32_t *>(whole(&wanted(arg[3], "lens"), "lens", at::kInt, {a.rows}, device));
      a.prompt_lens = static_cast<const int32_t *>(whole(given(arg[4], "prompt_lens"), "prompt_lens", at::kInt, {a.rows}, device));
      if (!a.tokens) a.lens = a.prompt_lens = nullptr; // no columns
    } else if (arg[3] != Py_None || arg[4] != Py_None) {
      throw Wrong{"tokens", "lengths without tokens"};
    }
    a.repetition = per_row(arg[5], "repetition", a.rows, device), a.frequency = per_row(arg[6], "frequency", a.rows, device);
    a.presence = per_row(arg[7], "presence", a.rows, device);
    if (!bias != !bias_ids) throw Wrong{"bias", "biases and their ids go together"};
    if (bias) {
      if (bias->dim() != 2) throw Wrong{"bias", "[row, place] is wanted"};
      const int64_t n = bias->size(1);
      a.bias = static_cast<const float *>(whole(bias, "bias", at::kFloat, {a.rows, n}, device));
      a.bias_ids = static_cast<const int32_t *>(whole(bias_ids, "bias_ids", at::kInt, {a.rows, n}, device));
      a.n_bias = int32_of(n, "bias");
    }
    if (allowed) {
      if (allowed->scalar_type() != at::kInt || allowed->dim() != 2) throw Wrong{"allowed", "int32 [row, word] is wanted"};
      const Matrix m = matrix_of(*allowed, "allowed", allowed->size(0), (a.vocab + 31) / 32, device);
      a.allowed = static_cast<const uint32_t *>(m.at), a.allowed_stride = m.stride, a.n_allowed = int32_of(allowed->size(0), "allowed");
      a.allowed_rows = static_cast<const int32_t *>(whole(allowed_rows, "allowed_rows", at::kInt, {a.rows}, device));
      if (!allowed_rows && a.n_allowed != a.rows) throw Wrong{"allowed", "a row for every row of the logits, or allowed_rows, is wanted"};
    } else if (allowed_rows) {
      throw Wrong{"allowed_rows", "allowed is wanted with it"};
    }
    Tensor made;
    if (!out) made = at::empty(logits.sizes(), logits.options());
    const Tensor &to = out ? *out : made;
    a.out = like(to, logits), a.out_stride = to.stride(0);
    if (const int code = hf_adjust_logits(&a, stream_of(arg[0]))) return failed(code, "hf_adjust_logits");
    written({out});
    return out ? again(arg[12]) : wrap(std::move(made));
  });
}

// (stream, logits, ids, logprobs, temperature, reverse, rest) -> (loss, norm, slopes)
PyObject *distill(PyObject *, PyObject *const *arg, Py_ssize_t n_args) {
  return guarded(n_args, 7, [&]() -> PyObject * {
    const Tensor &logits = wanted(arg[1], "logits"), &ids = wanted(arg[2], "top_ids"), &logprobs = wanted(arg[3], "top_logprobs");
    const hf_logits x = logits_of(logits, nullptr, real(arg[4]));
    const int device = logits.get_device();
    const c10::DeviceGuard current(logits.device());
    if (ids.dim() != 2) throw Wrong{"top_ids", "[row, place] is wanted"};
    const int64_t n = ids.size(1);
    hf_distillation a = {};
    a.ids = static_cast<const int32_t *>(whole(&ids, "top_ids", at::kInt, {x.rows, n}, device));
    a.logprobs = static_cast<const float *>(whole(&logprobs, "top_logprobs", at::kFloat, {x.rows, n}, device));
    a.n = int32_of(n, "top_ids"), a.reverse = (float)real(arg[5]);
    const int rest = PyObject_IsTrue(arg[6]);
    if (rest < 0) throw python_error();
    a.flags = rest ? HF_DISTILL_REST : 0;
    // A loss outlives the step and would hold the others: it lies by itself, unless all of them are few numbers (14 rows of 5004 f32, forward and gradient, 9.6 us for 10.1)
    const bool apart = x.rows * (n + 4) * 4 > 4096;
    Tensor own;
    Made made(logits);
    int loss = -1;
    if (apart) own = at::empty({x.rows}, logits.options().dtype(at::kFloat)), a.loss = static_cast<float *>(own.data_ptr());
    else loss = made.output(Py_None, "loss", at::kFloat, {x.rows}, &a.loss);
    const int norm = made.output(Py_None, "norm", at::kFloat, {x.rows, 2}, &a.norm), slopes = made.output(Py_None, "slopes", at::kFloat, {x.rows, n + 1}, &a.slopes);
    made.make();
    if (const int code = hf_top_distill(&x, &a, stream_of(arg[0]))) return failed(code, "hf_top_distill");
    return tuple_of({apart ? wrap(std::move(own)) : made.result(loss, Py_None), made.result(norm, Py_None), made.result(slopes, Py_None)});
  });
}

// (stream, logits, ids, norm, slopes, grad_loss, temperature, out) -> out
PyObject *distill_back(PyObject *, PyObject *const *arg, Py_ssize_t n_args) {
  return guarded(n_args, 8, [&]() -> PyObject * {
    const Tensor &logits = wanted(arg[1], "logits"), &ids = wanted(arg[2], "top_ids"), *out = given(arg[7], "out");
    const hf_logits x = logits_of(logits, nullptr, real(arg[6]));
    const int device = logits.get_device();
    const c10::DeviceGuard current(logits.device());
    if (ids.dim() != 2) throw Wrong{"top_ids", "[row, place] is wanted"};
    const int64_t n = ids.size(1);
    hf_distillation_grad g = {};
    g.ids = static_cast<const int32_t *>(whole(&ids, "top_ids", at::kInt, {x.rows, n}, device));
    g.norm = static_cast<const float *>(whole(&wanted(arg[3], "norm"), "norm", at::kFloat, {x.rows, 2}, device));
    g.slopes = static_cast<const float *>(whole(&wanted(arg[4], "slopes"), "slopes", at::kFloat, {x.rows, n + 1}, device));
    g.grad_loss = static_cast<const float *>(whole(&wanted(arg[5], "grad_loss"), "grad_loss", at::kFloat, {x.rows}, device));
    g.n = int32_of(n, "top_ids");
    Tensor made;
    if (!out) made = at::empty(logits.sizes(), logits.options());
    const Tensor &to = out ? *out : made;
    g.dlogits = like(to, logits), g.dlogits_stride = to.stride(0);
    if (const int code = hf_top_distill_back(&x, &g, stream_of(arg[0]))) return failed(code, "hf_top_distill_back");
    written({out});
    return out ? again(arg[7]) : wrap(std::move(made));
  });
}

// ---- pages ---------------------------------------------------------------------------------------------------------------

// A pool: its caches as bytes, and a tuple of their tensors.
struct Pool {
  hf_page_pool c;
  PyObject *tensors;
  Pool(PyObject *caches, PyObject *tuple) : c{}, tensors(tuple) {
    if (!PyBytes_Check(caches) || PyBytes_GET_SIZE(caches) % sizeof(hf_kv_cache) || !PyTuple_Check(tuple)) throw Wrong{"pool", "hf_kv_caches in bytes and their tensors are wanted"};
    c.caches = reinterpret_cast<const hf_kv_cache *>(PyBytes_AS_STRING(caches));
    c.n_caches = (int32_t)(PyBytes_GET_SIZE(caches) / sizeof(hf_kv_cache));
    if (c.n_caches < 1) throw Wrong{"pool", "at least one cache is wanted"};
  }
  int64_t pages() const { return c.caches[0].n_pages; }
  template <typename F> void each(const F &f) const {
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(tensors); ++i) f(wanted(PyTuple_GET_ITEM(tensors, i), "pool"));
  }
  // the GPU that all tensors are on has to be the pool's; `moves`: data are written, which takes no gradient
  void check(int device, bool moves) const {
    const Modes modes; // looked at once for all of them
    each([&](const Tensor &t) {
      if (!t.is_cuda() || t.get_device() != device) throw Wrong{"pool", "caches on the operands' GPU are wanted"};
      if (moves) without_gradient({{"pool", &t}}, modes);
    });
  }
  void moved() const {
    each([](const Tensor &t) { written({&t}); });
  }
};
const Tensor &on_gpu(PyObject *o, const char *name) {
  const Tensor &t = wanted(o, name);
  if (!t.is_cuda()) throw Wrong{name, "a tensor on the GPU is wanted"};
  return t;
}
const Tensor &table_of(PyObject *o) {
  const Tensor &t = on_gpu(o, "tables");
  if (t.dim() != 2) throw Wrong{"tables", "[row, page] is wanted"};
  return t;
}

// (caches, their tensors, stream, tables, lens, parents, refs, tables_out, lens_out, refs_out, workspace) -> (tables, lens, refs)
PyObject *fork(PyObject *, PyObject *const *arg, Py_ssize_t n_args) {
  return guarded(n_args, 11, [&]() -> PyObject * {
    const Pool pool(arg[0], arg[1]);
    const Tensor &tables = table_of(arg[3]), &parents = wanted(arg[5], "parents");
    const int device = tables.get_device();
    const c10::DeviceGuard current(tables.device());
    pool.check(device, true);
    if (parents.dim() != 1) throw Wrong{"parents", "[row] is wanted"};
    const int64_t rows = tables.size(0), width = tables.size(1), out = parents.size(0);
    hf_page_fork a = {};
    a.rows = int32_of(rows, "tables"), a.rows_out = int32_of(out, "parents"), a.width = int32_of(width, "tables");
    a.tables = static_cast<const int32_t *>(whole(&tables, "tables", at::kInt, {rows, width}, device));
    a.lens = static_cast<const int32_t *>(whole(&wanted(arg[4], "lens"), "lens", at::kInt, {rows}, device));
    a.parents = static_cast<const int32_t *>(whole(&parents, "parents", at::kInt, {out}, device));
    a.refs = static_cast<const int32_t *>(whole(&wanted(arg[6], "refs"), "refs", at::kInt, {pool.pages()}, device));
    Made made(tables);
    const int new_tables = made.output(arg[7], "tables_out", at::kInt, {out, width}, &a.tables_out), new_lens = made.output(arg[8], "lens_out", at::kInt, {out}, &a.lens_out);
    const int new_refs = made.output(arg[9], "refs_out", at::kInt, {pool.pages()}, &a.refs_out);
    const size_t size = hf_fork_pages_workspace_bytes(&pool.c, &a);
    if (size == (size_t)-1) return failed(HF_EINVAL, "hf_fork_pages_workspace_bytes");
    made.make(a, size, arg[10]);
    if (const int code = hf_fork_pages(&pool.c, &a, stream_of(arg[2]))) return failed(code, "hf_fork_pages");
    pool.moved();
    written({given(arg[7], "tables_out"), given(arg[8], "lens_out"), given(arg[9], "refs_out"), given(arg[10], "workspace")});
    return tuple_of({made.result(new_tables, arg[7]), made.result(new_lens, arg[8]), made.result(new_refs, arg[9])});
  });
}

// (caches, their tensors, stream, tables, lens, counts, refs, most, tables_out, lens_out, slots, refs_out, workspace) -> (tables, lens, slots, refs)
PyObject *grow(PyObject *, PyObject *const *arg, Py_ssize_t n_args) {
  return guarded(n_args, 13, [&]() -> PyObject * {
    const Pool pool(arg[0], arg[1]);
    const Tensor &tables = table_of(arg[3]);
    const int device = tables.get_device();
    const c10::DeviceGuard current(tables.device());
    pool.check(device, false);
    const int64_t rows = tables.size(0), width = tables.size(1), most = number(arg[7]);
    if (most < 0) throw Wrong{"most", "a number of tokens is wanted"};
    hf_page_grow a = {};
    a.rows = int32_of(rows, "tables"), a.width = int32_of(width, "tables"), a.most = int32_of(most, "most");
    a.tables = static_cast<const int32_t *>(whole(&tables, "tables", at::kInt, {rows, width}, device));
    a.lens = static_cast<const int32_t *>(whole(&wanted(arg[4], "lens"), "lens", at::kInt, {rows}, device));
    a.counts = static_cast<const int32_t *>(whole(&wanted(arg[5], "counts"), "counts", at::kInt, {rows}, device));
    a.refs = static_cast<const int32_t *>(whole(&wanted(arg[6], "refs"), "refs", at::kInt, {pool.pages()}, device));
    Made made(tables);
    const int new_tables = made.output(arg[8], "tables_out", at::kInt, {rows, width}, &a.tables_out), new_lens = made.output(arg[9], "lens_out", at::kInt, {rows}, &a.lens_out);
    const int new_slots = made.output(arg[10], "slots", at::kLong, {rows, most}, &a.slots), new_refs = made.output(arg[11], "refs_out", at::kInt, {pool.pages()}, &a.refs_out);
    const size_t size = hf_grow_pages_workspace_bytes(&pool.c, &a);
    if (size == (size_t)-1) return failed(HF_EINVAL, "hf_grow_pages_workspace_bytes");
    made.make(a, size, arg[12]);
    if (const int code = hf_grow_pages(&pool.c, &a, stream_of(arg[2]))) return failed(code, "hf_grow_pages");
    written({given(arg[8], "tables_out"), given(arg[9], "lens_out"), given(arg[10], "slots"), given(arg[11], "refs_out"), given(arg[12], "workspace")});
    return tuple_of({made.result(new_tables, arg[8]), made.result(new_lens, arg[9]), made.result(new_slots, arg[10]), made.result(new_refs, arg[11])});
  });
}

// (caches, their tensors, stream, refs, tables as a tuple, tables_out as a tuple of tensors or None, refs_out, workspace) -> (tables as a tuple, refs, places, live)
PyObject *compact(PyObject *, PyObject *const *arg, Py_ssize_t n_args) {
  return guarded(n_args, 8, [&]() -> PyObject * {
    const Pool pool(arg[0], arg[1]);
    const Tensor &refs = on_gpu(arg[3], "refs");
    const int device = refs.get_device();
    const c10::DeviceGuard current(refs.device());
    pool.check(device, true);
    if (!PyTuple_Check(arg[4]) || !PyTuple_Check(arg[5]) || PyTuple_GET_SIZE(arg[4]) != PyTuple_GET_SIZE(arg[5])) throw Wrong{"tables_out", "as many as tables are wanted"};
    const Py_ssize_t n = PyTuple_GET_SIZE(arg[4]);
    if (n > HF_MAX_TABLES) throw Wrong{"tables", "at most HF_MAX_TABLES at a time"};
    hf_page_compact a = {};
    a.refs = static_cast<const int32_t *>(whole(&refs, "refs", at::kInt, {pool.pages()}, device));
    Made made(refs);
    int new_tables[HF_MAX_TABLES];
    for (Py_ssize_t i = 0; i < n; ++i) {
      const Tensor &t = on_gpu(PyTuple_GET_ITEM(arg[4], i), "tables");
      if (t.get_device() != device || t.scalar_type() != at::kInt || !t.is_contiguous()) throw Wrong{"tables", "contiguous int32 tensors on one GPU are wanted"};
      a.entries[i] = static_cast<const int32_t *>(t.data_ptr());
      a.n_entries[i] = t.numel();
      new_tables[i] = made.output(PyTuple_GET_ITEM(arg[5], i), "tables_out", at::kInt, t.sizes(), &a.entries_out[i]);
    }
    const int new_refs = made.output(arg[6], "refs_out", at::kInt, {pool.pages()}, &a.refs_out);
    const int places = made.output(Py_None, "places", at::kInt, {pool.pages()}, &a.places), live = made.output(Py_None, "live", at::kInt, {}, &a.live);
    const size_t size = hf_compact_pages_workspace_bytes(&pool.c, &a);
    if (size == (size_t)-1) return failed(HF_EINVAL, "hf_compact_pages_workspace_bytes");
    made.make(a, size, arg[7]);
    if (const int code = hf_compact_pages(&pool.c, &a, stream_of(arg[2]))) return failed(code, "hf_compact_pages");
    pool.moved();
    written({given(arg[6], "refs_out"), given(arg[7], "workspace")});
    PyObject *tables = PyTuple_New(n);
    if (!tables) return nullptr;
    for (Py_ssize_t i = 0; i < n; ++i) {
      PyObject *o = PyTuple_GET_ITEM(arg[5], i);
      written({given(o, "tables_out")});
      PyTuple_SET_ITEM(tables, i, made.result(new_tables[i], o));
    }
    return tuple_of({tables, made.result(new_refs, arg[6]), made.result(places, Py_None), made.result(live, Py_None)});
  });
}

PyMethodDef g_methods[] = {{"adjust", fast(adjust), METH_FASTCALL, nullptr},   {"distill", fast(distill), METH_FASTCALL, nullptr},
                           {"distill_back", fast(distill_back), METH_FASTCALL, nullptr}, {"fork", fast(fork), METH_FASTCALL, nullptr},
                           {"grow", fast(grow), METH_FASTCALL, nullptr},       {"compact", fast(compact), METH_FASTCALL, nullptr},
                           {"set_error", set_error, METH_O, nullptr},          {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_steps", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__steps(void) { return PyModule_Create(&g_module); }
