// Append of new tokens' keys and values to a paged cache, with the position rotation on the way.
//
//   pair (a, b) of a head at position p, pair index i:  (a cos[p,i] - b sin[p,i],  b cos[p,i] + a sin[p,i])
//
// Every byte is read once and written once, so HBM is the bound; the rotation costs six operations a pair.  A
// workgroup takes one token: its lanes lie over the pairs of a head and then over the heads, so that a lane needs the cosines and
// sines of its pairs once for all the heads that it serves (they are as long as a head's data and would otherwise be read again, from L2, for
// each), and a wavefront reads and writes whole heads.  A lane moves two vectors of up to 16 bytes, one
// of each half of its pairs.  8192 tokens of 32 heads of 128 (q, k and v, bf16): 76 us, 5.05 TB/s read and written (non-temporal stores level, system-scope
// ones 117 us, two or eight heads in flight level or slower); up to some 256 tokens 3 us, what a kernel takes to start and read four things one after another.
#include <hip/hip_runtime.h>

#include "rollout_kernels.hpp"

namespace hf {

namespace {

constexpr int kThreads = 256;

template <typename T, int kVec> struct alignas(sizeof(T) * kVec) Vec {
  T e[kVec];
};

struct AppendParams {
  hf_append a;
  void *cache_k, *cache_v;
  int64_t page_stride, head_stride, token_stride, n_slots;
  int32_t n_kv_heads, head_dim, page_shift, lane_shift, chunks;
};

constexpr int kRows = 4; // heads that a lane has in flight

template <typename T, int kVec, bool kInterleaved> __global__ __launch_bounds__(kThreads) void append_kv(AppendParams p) {
  typedef Vec<T, kVec> V;
  const hf_append &a = p.a;
  const int64_t t = blockIdx.x;
  const int chunk = threadIdx.x & ((1 << p.lane_shift) - 1), step = kThreads >> p.lane_shift;
  const int n_q = a.q ? a.n_q_heads : 0, n_k = n_q + p.n_kv_heads, n_rows = n_k + p.n_kv_heads;
  const int turned = a.rot_dim / (2 * kVec); // chunks of pairs; the others are copied
  const int64_t slot = a.slots[t];
  const int32_t at = a.rot_dim ? a.positions[t] : 0;
  const bool live = slot >= 0 && slot < p.n_slots && (a.rot_dim == 0 || (at >= 0 && at < a.n_positions));
  if (!live || chunk >= p.chunks) return;
  const bool turns = chunk < turned;
  // where the two vectors of a rotated head are; a value head has its in order
  const int in_order = 2 * kVec * chunk;
  const int first = turns && !kInterleaved ? kVec * chunk : in_order;
  const int second = turns && !kInterleaved ? a.rot_dim / 2 + kVec * chunk : in_order + kVec;
  float c[kVec], s[kVec];
  if (turns) {
    const int64_t row = (int64_t)at * (a.rot_dim / 2) + kVec * chunk;
#pragma unroll
    for (int e = 0; e < kVec; ++e) c[e] = a.cos[row + e], s[e] = a.sin[row + e];
  }
  const int64_t place = (slot >> p.page_shift) * p.page_stride + (slot & ((1 << p.page_shift) - 1)) * p.token_stride;

  for (int row0 = threadIdx.x >> p.lane_shift; row0 < n_rows; row0 += kRows * step) {
    V x[kRows], y[kRows];
    T *to[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int row = row0 + r * step;
      if (row >= n_rows) break;
      const T *from;
      if (row < n_q) {
        from = static_cast<const T *>(a.q) + t * a.q_stride + row * a.q_head_stride;
        to[r] = static_cast<T *>(a.q_out) + t * a.q_out_stride + row * a.q_out_head_stride;
      } else if (row < n_k) {
        from = static_cast<const T *>(a.k) + t * a.k_stride + (row - n_q) * a.k_head_stride;
        to[r] = static_cast<T *>(p.cache_k) + place + (row - n_q) * p.head_stride;
      } else {
        from = static_cast<const T *>(a.v) + t * a.v_stride + (row - n_k) * a.v_head_stride;
        to[r] = static_cast<T *>(p.cache_v) + place + (row - n_k) * p.head_stride;
      }
      const bool value = row >= n_k;
      const int i = value ? in_order : first, j = value ? in_order + kVec : second;
      x[r] = *reinterpret_cast<const V *>(from + i);
      if (j < p.head_dim) y[r] = *reinterpret_cast<const V *>(from + j);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int row = row0 + r * step;
      if (row >= n_rows) break;
      const bool value = row >= n_k;
      const int i = value ? in_order : first, j = value ? in_order + kVec : second;
      V u = x[r], w = y[r];
      if (turns && !value) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          // element e of the chunk's 2 * kVec: its pair's halves are apart in two vectors, or beside one another
          const float f = (float)(kInterleaved ? (2 * e < kVec ? x[r].e[2 * e % kVec] : y[r].e[2 * e % kVec]) : x[r].e[e]);
          const float g = (float)(kInterleaved ? (kVec == 1 ? y[r].e[0] : 2 * e < kVec ? x[r].e[(2 * e + 1) % kVec] : y[r].e[(2 * e + 1) % kVec]) : y[r].e[e]);
          const T h = (T)(f * c[e] - g * s[e]), l = (T)(g * c[e] + f * s[e]);
          if (!kInterleaved || kVec == 1) u.e[e] = h, w.e[e] = l;
          else if (2 * e < kVec) u.e[2 * e % kVec] = h, u.e[(2 * e + 1) % kVec] = l;
          else w.e[2 * e % kVec] = h, w.e[(2 * e + 1) % kVec] = l;
        }
      }
      *reinterpret_cast<V *>(to[r] + i) = u;
      if (j < p.head_dim) *reinterpret_cast<V *>(to[r] + j) = w;
    }
  }
}

template <typename T, int kVec> hipError_t launch(const AppendParams &p, hipStream_t st) {
  const dim3 grid(p.a.n_tokens);
  if (p.a.flags & HF_ROT_INTERLEAVED) return enqueue_kernel(append_kv<T, kVec, true>, grid, kThreads, st, p);
  return enqueue_kernel(append_kv<T, kVec, false>, grid, kThreads, st, p);
}

template <typename T> hipError_t launch_vec(const AppendParams &p, int vec, hipStream_t st) {
  switch (vec) {
  case 8: return launch<T, 8>(p, st);
  case 4: return launch<T, 4>(p, st);
  case 2: return launch<T, 2>(p, st);
  default: return launch<T, 1>(p, st);
  }
}

int shift_of(int64_t n) { // smallest s with 2^s >= n
  int s = 0;
  while ((int64_t(1) << s) < n) ++s;
  return s;
}

} // namespace

int launch_append(const hf_kv_cache &cache, const hf_append &args, int vec, void *stream) {
  const int chunks = (cache.head_dim + 2 * vec - 1) / (2 * vec);
  const AppendParams p = {args, cache.k, cache.v, cache.page_stride, cache.head_stride, cache.token_stride,
                          cache.n_pages * cache.page_tokens, cache.n_kv_heads, cache.head_dim, shift_of(cache.page_tokens), shift_of(chunks), chunks};
  hipStream_t st = static_cast<hipStream_t>(stream);
  return (int)(cache.dtype == HF_BF16 ? launch_vec<__bf16>(p, vec, st) : launch_vec<_Float16>(p, vec, st));
}

} // namespace hf
