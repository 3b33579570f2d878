// What the C entry points of the rollout operators check on the host: strides, places in memory and overlaps, caches and logits.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "hfreshard.h"
#include "kernels.hpp"

namespace hf::check {

inline constexpr unsigned __int128 kMost = (unsigned __int128)1 << 60; // elements that a tensor may span

struct Dim {
  int64_t n, stride;
};

inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// elements from the first to past the last of a tensor whose innermost `inner` are contiguous; 0 = a negative stride or a span beyond kMost
template <size_t kN> int64_t span(const Dim (&dims)[kN], int64_t inner) {
  unsigned __int128 all = inner;
  for (const Dim &d : dims) {
    if (d.n == 0) continue;
    if (d.stride < 0) return 0;
    all += (unsigned __int128)(d.n - 1) * (uint64_t)d.stride;
    if (all > kMost) return 0;
  }
  return (int64_t)all;
}

// whether no two elements of it share a place (the dimensions nest in some order)
template <size_t kN> bool separate(const Dim (&dims)[kN], int64_t inner) {
  unsigned __int128 need = inner;
  bool used[kN] = {};
  for (size_t k = 0; k < kN; ++k) { // by ascending stride
    size_t best = kN;
    for (size_t i = 0; i < kN; ++i)
      if (!used[i] && (best == kN || dims[i].stride < dims[best].stride)) best = i;
    used[best] = true;
    if (dims[best].n <= 1) continue;
    if ((unsigned __int128)dims[best].stride < need) return false;
    need += (unsigned __int128)(dims[best].n - 1) * (uint64_t)dims[best].stride;
  }
  return true;
}

// Where a tensor lies, in bytes: `inner` of them in a row at every step of the dimensions, all from `begin` to `end` (both 0: nowhere).
struct Place {
  uintptr_t begin = 0, end = 0;
  int64_t inner = 0;
  Dim dims[3] = {{1, 0}, {1, 0}, {1, 0}};
};
inline Place array(const void *at, int64_t n, int64_t size) {
  Place p;
  if (!at || n <= 0) return p;
  p.inner = n > (INT64_MAX >> 3) / size ? INT64_MAX >> 3 : n * size;
  p.begin = reinterpret_cast<uintptr_t>(at), p.end = p.begin + p.inner;
  return p;
}
// of a tensor whose span() is known to be in contract
template <size_t kN> Place place(const void *at, const Dim (&dims)[kN], int64_t inner, int64_t size) {
  Place p = array(at, inner, size);
  for (size_t i = 0; i < kN; ++i) {
    if (dims[i].n == 0) return Place{};
    p.dims[i] = {dims[i].n, dims[i].stride * size};
    p.end += (dims[i].n - 1) * p.dims[i].stride;
  }
  return at ? p : Place{};
}

// Whether the runs of bytes that begin `apart` from one another and at any whole numbers of steps more meet; steps are by descending stride.
inline bool meet_steps(__int128 apart, int64_t a_inner, int64_t b_inner, const Dim *steps, const int64_t (&a_n)[3], const int64_t (&b_n)[3], int i) {
  while (i < 3 && a_n[i] <= 1 && b_n[i] <= 1) ++i;
  if (i == 3) return -b_inner < apart && apart < a_inner;
  const int64_t stride = steps[i].stride;
  __int128 j = -apart / stride; // what is below reaches no further than a step: at most the three nearest ones bring them together
  for (__int128 k = j - 1; k <= j + 1; ++k)
    if (k >= -(a_n[i] - 1) && k <= b_n[i] - 1 && meet_steps(apart + k * stride, a_inner, b_inner, steps, a_n, b_n, i + 1)) return true;
  return false;
}

// Whether two tensors share a byte.  Exact where neither reaches into the other's range, and where their strides are alike (slices of one tensor, such as
// the queries and keys of one projection); otherwise tensors whose ranges meet are taken to.
inline bool overlap(const Place &a, const Place &b) { // (an empty place is before all others)
  if (a.begin >= b.end || b.begin >= a.end) return false;
  Dim steps[3] = {};
  int64_t a_n[3], b_n[3];
  for (int i = 0; i < 3; ++i) {
    const Dim &d = a.dims[i], &e = b.dims[i];
    if (d.n > 1 && e.n > 1 && d.stride != e.stride) return true;
    steps[i] = {i, d.n > 1 ? d.stride : e.n > 1 ? e.stride : 0};
  }
  std::sort(steps, steps + 3, [](const Dim &d, const Dim &e) { return d.stride > e.stride; });
  for (int i = 0; i < 3; ++i) a_n[i] = a.dims[steps[i].n].n, b_n[i] = b.dims[steps[i].n].n;
  int64_t reach = std::max(a.inner, b.inner); // nested: what lies below a step is within it
  for (int i = 2; i >= 0; --i) {
    const int64_t n = std::max(a_n[i], b_n[i]);
    if (n <= 1) continue;
    if (steps[i].stride < reach) return true;
    reach += (n - 1) * steps[i].stride;
  }
  return meet_steps((__int128)b.begin - (__int128)a.begin, a.inner, b.inner, steps, a_n, b_n, 0);
}
// the first of the outputs that lies in an input or in another output, by its name; null: none
struct Output {
  const char *what;
  Place place;
};
template <size_t kN> const char *first_overlap(const Output (&outputs)[kN], std::initializer_list<Place> inputs) {
  for (size_t i = 0; i < kN; ++i) {
    for (const Place &p : inputs)
      if (overlap(outputs[i].place, p)) return outputs[i].what;
    for (size_t j = 0; j < i; ++j)
      if (overlap(outputs[i].place, outputs[j].place)) return outputs[i].what;
  }
  return nullptr;
}

// whether a tensor's vectors of `vec` 2-byte elements are aligned wherever they begin
template <size_t kN> bool divides(const void *p, const Dim (&dims)[kN], int vec) {
  if (!aligned(p, 2 * vec)) return false;
  for (const Dim &d : dims)
    if (d.n > 1 && d.stride % vec) return false;
  return true;
}

inline int check_cache(const hf_kv_cache *c) {
  if (!c) return set_error(HF_EINVAL, "null cache");
  if (!c->k || !c->v) return set_error(HF_EINVAL, "null cache buffer");
  if (c->k == c->v) return set_error(HF_EINVAL, "keys and values lie in the same place");
  if (c->dtype != HF_BF16 && c->dtype != HF_F16) return set_error(HF_EINVAL, "a cache is HF_BF16 or HF_F16");
  if (!aligned(c->k, 2) || !aligned(c->v, 2)) return set_error(HF_EINVAL, "cache buffers must be aligned to their elements");
  if (c->n_kv_heads < 1) return set_error(HF_EINVAL, "n_kv_heads must be positive");
  if (c->head_dim < 1 || c->head_dim > 256) return set_error(HF_EINVAL, "head_dim must be in [1, 256]");
  if (c->page_tokens < 4 || c->page_tokens > 65536 || (c->page_tokens & (c->page_tokens - 1)))
    return set_error(HF_EINVAL, "page_tokens must be a power of two in [4, 65536]");
  if (c->n_pages < 1 || c->n_pages > INT32_MAX) return set_error(HF_EINVAL, "n_pages must be in [1, 2^31 - 1]");
  const Dim dims[] = {{c->n_pages, c->page_stride}, {c->n_kv_heads, c->head_stride}, {c->page_tokens, c->token_stride}};
  if (!span(dims, c->head_dim)) return set_error(HF_EINVAL, "cache strides are negative or span too much");
  if (!separate(dims, c->head_dim)) return set_error(HF_EINVAL, "cache strides put two tokens in one place");
  return HF_OK;
}

inline int check_logits(const hf_logits *in) {
  if (!in) return set_error(HF_EINVAL, "null arguments");
  if (in->dtype != HF_BF16 && in->dtype != HF_F16 && in->dtype != HF_F32) return set_error(HF_EINVAL, "unknown type of logits");
  if (in->rows < 0) return set_error(HF_EINVAL, "negative size");
  if (in->vocab < 1 || in->vocab > (1 << 30)) return set_error(HF_EINVAL, "vocab must be in [1, 2^30]");
  if (!(in->inv_temperature > 0) || !std::isfinite(in->inv_temperature)) return set_error(HF_EINVAL, "inv_temperature must be positive and finite");
  if (in->rows == 0) return HF_OK;
  if (!in->logits) return set_error(HF_EINVAL, "null logits");
  const Dim dims[] = {{in->rows, in->row_stride}};
  if (!span(dims, in->vocab)) return set_error(HF_EINVAL, "row_stride is negative or spans too much");
  if (!aligned(in->logits, in->dtype == HF_F32 ? 4 : 2)) return set_error(HF_EINVAL, "logits must be aligned to their elements");
  if (in->targets && in->target_bytes != 4 && in->target_bytes != 8) return set_error(HF_EINVAL, "target_bytes must be 4 or 8");
  if (in->targets && !aligned(in->targets, in->target_bytes)) return set_error(HF_EINVAL, "targets must be aligned to their elements");
  return HF_OK;
}

inline int launched(int e) {
  if (e != 0) return set_error(HF_EHIP, hipGetErrorString(static_cast<hipError_t>(e)));
  return HF_OK;
}

} // namespace hf::check
