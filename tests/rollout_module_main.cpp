// The native module of rollout.py over a stand-in for the library and for the GPUs, so that what it does with devices can be seen on a machine without any:
// tensors that say they are on a GPU, torch's own stand-in for the current device, and library calls that note where they were made.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/FakeGuardImpl.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdlib>
#include <vector>

using Guard = c10::impl::FakeGuardImpl<c10::DeviceType::CUDA>;
C10_REGISTER_GUARD_IMPL(CUDA, Guard)

static at::Tensor stand_in(at::IntArrayRef shape, at::ScalarType type, int device) {
  int64_t n = 1;
  for (const int64_t s : shape) n *= s;
  const size_t bytes = n * c10::elementSize(type);
  void *p = std::calloc(bytes + 64, 1);
  c10::Storage storage(c10::make_intrusive<c10::StorageImpl>(c10::StorageImpl::use_byte_size_t(), bytes, c10::DataPtr(p, p, std::free, c10::Device(c10::kCUDA, device)),
                                                             nullptr, false));
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(std::move(storage), c10::DispatchKeySet(c10::DispatchKey::CUDA), c10::scalarTypeToTypeMeta(type));
  t.unsafeGetTensorImpl()->set_sizes_contiguous(shape);
  return t;
}
namespace at {
inline Tensor empty_stand_in(IntArrayRef shape, const TensorOptions &o) {
  return stand_in(shape, c10::typeMetaToScalarType(o.dtype()), o.device().index());
}
} // namespace at

#define empty empty_stand_in // (every header that says it is in already)
#undef PY_SSIZE_T_CLEAN
#include "rollout_torch.cpp"
#undef empty

struct Call {
  const char *name;
  int device;
  void *stream;
};
static std::vector<Call> g_calls;
static int note(const char *name, void *stream) {
  g_calls.push_back({name, Guard::getDeviceIndex(), stream});
  return HF_OK;
}

extern "C" {
int hf_append_kv(const hf_kv_cache *, const hf_append *, void *s) { return note("hf_append_kv", s); }
size_t hf_attend_workspace_bytes(const hf_kv_cache *, const hf_attention *) { return 512; }
int hf_attend(const hf_kv_cache *, const hf_attention *, void *s) { return note("hf_attend", s); }
int hf_token_logprobs(const hf_logits *, const hf_logprobs *, void *s) { return note("hf_token_logprobs", s); }
int hf_token_logprobs_back(const hf_logits *, const hf_logprobs_grad *, void *s) { return note("hf_token_logprobs_back", s); }

// for ctypes.PyDLL
__attribute__((visibility("default"))) PyObject *stand_in_tensor(PyObject *shape, int type, int device) {
  std::vector<int64_t> s;
  for (Py_ssize_t i = 0; i < PyTuple_Size(shape); ++i) s.push_back(PyLong_AsLongLong(PyTuple_GetItem(shape, i)));
  return THPVariable_Wrap(stand_in(s, static_cast<at::ScalarType>(type), device));
}
__attribute__((visibility("default"))) PyObject *calls() { // and forgets them
  PyObject *list = PyList_New(0);
  for (const Call &c : g_calls) {
    PyObject *t = Py_BuildValue("(siK)", c.name, c.device, (unsigned long long)(uintptr_t)c.stream);
    PyList_Append(list, t);
    Py_DECREF(t);
  }
  g_calls.clear();
  return list;
}
__attribute__((visibility("default"))) int current_device() { return Guard::getDeviceIndex(); }
}
