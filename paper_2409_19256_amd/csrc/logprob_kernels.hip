// Log probabilities of given tokens, the entropy and the likeliest tokens of rows of logits, and the gradient of the first two.
//
//   y = x / temperature;  m = max y;  z = sum e^(y-m);  lse = m + ln z;  logprob = y_t - lse;  H = ln z - sum e^(y-m) (y-m) / z
//   dx_j = ([j = t] g - p_j (g + h (ln p_j + H))) / temperature
//
// The forward pass reads every logit once and writes a few numbers a row; the gradient reads and writes each once.  HBM is
// the bound: at 2 bytes an element there is room for about fourteen vector operations on each, and the forward pass needs nine (a base-2
// exponential counts as four).  A workgroup takes a row; every lane keeps its own running maximum, sum and weighted sum over its vectors and
// they are merged once at the end.
//
// The likeliest tokens come out of the same pass: besides its maximum a lane remembers in which of its vectors it first met it.
// The top_n-th largest of 64 groups' maxima bounds the top_n-th largest element from below, so only lanes whose own maximum reaches that
// bound can hold an answer; they, about top_n of them, read their vectors again (from L2) and hand over what reaches the bound.  Keys are value and
// position together, so they are all different and ties fall to the lower id by themselves.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "rollout_kernels.hpp"

namespace hf {

namespace {

constexpr int kWave = 64;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kCandidates = 1024; // room for what reaches the bound; more go through find_by_rounds

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T> constexpr int kVec = 16 / sizeof(T); // elements of a vector

// rows begin at any element, so the address of a vector is a multiple of the element's size and no more
template <typename T> struct Vector {
  typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
  typedef type any __attribute__((aligned(sizeof(T))));
};
template <typename T> __device__ __forceinline__ typename Vector<T>::type load_vec(const T *p) { return *reinterpret_cast<const typename Vector<T>::any *>(p); }

// the order of floats as the order of unsigned numbers; -0 is 0, and every NaN comes last
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  return x != x ? 0xFFFFFFFEu : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
// larger value first, then the lower index
__device__ __forceinline__ uint64_t key_of(float x, uint32_t index) { return (uint64_t)order_of(x) << 32 | (0xFFFFFFFFu - index); }

struct Logits {
  const void *data, *targets;
  int64_t row_stride;
  int32_t vocab, target_bytes;
  float inv_temperature;
};

__device__ __forceinline__ int64_t target_of(const Logits &in, int64_t row) {
  return in.target_bytes == 8 ? static_cast<const int64_t *>(in.targets)[row] : static_cast<const int32_t *>(in.targets)[row];
}

// max, sum of exponentials and their sum weighted by the distance from the max, of base 2
struct Stats {
  float m, s, u;
};
// `to` moved to a larger maximum
__device__ __forceinline__ void rebase(Stats &st, float m, float c) {
  if (m > st.m) {
    const float d = st.m == -INFINITY ? 0.f : (st.m - m) * c; // before the first element there is nothing to move
    const float down = __builtin_amdgcn_exp2f(d);
    st.u = st.s > 0 ? down * fmaf(fmaxf(d, -200.f), st.s, st.u) : st.u;
    st.s *= down;
    st.m = m;
  }
}
__device__ __forceinline__ Stats merge(Stats a, Stats b, float c) {
  const float m = fmaxf(a.m, b.m);
  rebase(a, m, c);
  rebase(b, m, c);
  return {m, a.s + b.s, a.u + b.u};
}
__device__ __forceinline__ Stats merge_wave(Stats st, float c) {
#pragma unroll
  for (int d = kWave / 2; d; d /= 2) st = merge(st, {__shfl_xor(st.m, d), __shfl_xor(st.s, d), __shfl_xor(st.u, d)}, c);
  return st;
}

// elements of a group of vectors join the statistics; c = log2(e) / temperature
template <int kN> __device__ __forceinline__ void join(Stats &st, const float (&x)[kN], float top, float c) {
  rebase(st, top, c);
  const float at = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    const float d = (x[i] - at) * c;
    const float e = __builtin_amdgcn_exp2f(d); // NaN comes through here
    st.s += e;
    st.u = fmaf(e, fmaxf(d, -200.f), st.u); // 0 * -inf would be NaN, and 2^-200 is 0
  }
}

template <int kThreads> __device__ __forceinline__ uint64_t block_max(uint64_t key, uint64_t *shared) {
#pragma unroll
  for (int d = kWave / 2; d; d /= 2) key = max(key, (uint64_t)__shfl_xor((unsigned long long)key, d));
  if constexpr (kThreads > kWave) {
    __syncthreads();
    if (threadIdx.x % kWave == 0) shared[threadIdx.x / kWave] = key;
    __syncthreads();
    key = shared[0];
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) key = max(key, shared[w]);
  }
  return key;
}

// The top_n largest keys one after another, a pass over the row for each: for rows of which more than kCandidates elements reach the bound.
template <typename T, int kThreads, typename F>
__device__ void find_by_rounds(const T *row, int vocab, int top_n, F logprob_of, int32_t *ids, float *values, uint64_t *shared) {
  uint64_t below = ~0ull;
  for (int n = 0; n < top_n; ++n) {
    uint64_t best = 0;
    for (int i = threadIdx.x; i < vocab; i += kThreads) {
      const uint64_t key = key_of((float)row[i], i);
      if (key < below && key > best) best = key;
    }
    below = block_max<kThreads>(best, shared);
    if (threadIdx.x == 0) {
      if (ids) ids[n] = 0xFFFFFFFFu - (uint32_t)below;
      if (values) values[n] = logprob_of(value_of(below >> 32));
    }
  }
}

template <typename T, int kThreads, bool kTop> __global__ __launch_bounds__(kThreads) void token_logprobs(Logits in, hf_logprobs out) {
  constexpr int kWaves = kThreads / kWave, kV = kVec<T>, kAhead = 4;
  __shared__ Stats stats[kWaves];
  __shared__ uint64_t keys[kTop ? kThreads : 1], found[kTop ? kCandidates : 1], bound_key;
  __shared__ uint32_t n_found;
  const int64_t r = blockIdx.x;
  const int t = threadIdx.x, vocab = in.vocab;
  const int64_t target = in.targets ? target_of(in, r) : 0;
  if (target < 0 || target >= vocab) {
    if (t == 0) {
      if (out.logprob) out.logprob[r] = 0;
      if (out.entropy) out.entropy[r] = 0;
      if (out.lse) out.lse[r] = 0;
      if (out.norm) out.norm[2 * r] = out.norm[2 * r + 1] = 0;
    }
    if constexpr (kTop)
      if (t < out.top_n) {
        if (out.top_ids) out.top_ids[r * out.top_n + t] = -1;
        if (out.top_logprobs) out.top_logprobs[r * out.top_n + t] = 0;
      }
    return;
  }
  const T *row = static_cast<const T *>(in.data) + r * in.row_stride;
  const float c = in.inv_temperature * kLog2e;
  const int n_vec = vocab / kV; // whole ones
  Stats st = {-INFINITY, 0, 0};
  float best = -INFINITY;      // the lane's largest element
  uint32_t best_at = 0xFFFFFFFFu; // and the vector that had it first; none: no vectors
  const auto add = [&](const float(&x)[kV], int at) {
    float top = x[0];
#pragma unroll
    for (int e = 1; e < kV; ++e) top = fmaxf(top, x[e]);
    if constexpr (kTop)
      if (top > best || best_at == 0xFFFFFFFFu) best = top, best_at = at;
    join<kV>(st, x, top, c);
  };
  int i = t;
  for (; i + (kAhead - 1) * kThreads < n_vec; i += kAhead * kThreads) {
    typename Vector<T>::type v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v[k] = load_vec(row + (int64_t)(i + k * kThreads) * kV);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      float x[kV];
#pragma unroll
      for (int e = 0; e < kV; ++e) x[e] = (float)v[k][e];
      add(x, i + k * kThreads);
    }
  }
  for (; i < n_vec; i += kThreads) {
    const typename Vector<T>::type v = load_vec(row + (int64_t)i * kV);
    float x[kV];
#pragma unroll
    for (int e = 0; e < kV; ++e) x[e] = (float)v[e];
    add(x, i);
  }
  if (i == n_vec && n_vec * kV < vocab) { // the vector that the row ends in
    float x[kV];
#pragma unroll
    for (int e = 0; e < kV; ++e) x[e] = n_vec * kV + e < vocab ? (float)row[n_vec * kV + e] : -INFINITY;
    add(x, i);
  }

  st = merge_wave(st, c);
  if constexpr (kWaves > 1) {
    if (t % kWave == 0) stats[t / kWave] = st;
  }
  const uint64_t mine = kTop && best_at != 0xFFFFFFFFu ? key_of(best, best_at) : 0;
  if constexpr (kTop) {
    keys[t] = mine;
    if (t == 0) n_found = 0;
  }
  if constexpr (kWaves > 1 || kTop) __syncthreads();
  if constexpr (kWaves > 1) {
    st = stats[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) st = merge(st, stats[w], c);
  }
  // of base e: lse = top + log_z
  const float top = st.m == -INFINITY ? 0.f : st.m * in.inv_temperature, log_z = __builtin_amdgcn_logf(st.s) * kLn2;
  const auto logprob_of = [&](float x) { // nearer than x * inv_temperature - lse, whose terms are rounded where they are large
    return x == -INFINITY && st.s == st.s ? -INFINITY : (x - (st.m == -INFINITY ? 0.f : st.m)) * in.inv_temperature - log_z;
  };
  if (t == 0) {
    if (out.lse) out.lse[r] = top + log_z;
    if (out.norm) out.norm[2 * r] = st.m, out.norm[2 * r + 1] = log_z;
    if (out.entropy) out.entropy[r] = st.s == 0 ? 0.f : log_z - st.u / st.s * kLn2;
    if (out.logprob) out.logprob[r] = logprob_of((float)row[target]);
  }
  if constexpr (kTop) {
    int32_t *ids = out.top_ids ? out.top_ids + r * out.top_n : nullptr;
    float *values = out.top_logprobs ? out.top_logprobs + r * out.top_n : nullptr;
    if (t < kWave) {
      uint64_t key = keys[t];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) key = max(key, keys[t + w * kWave]);
      int rank = 0;
      for (int k = 0; k < kWave; ++k) {
        const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)key, k), hi = __builtin_amdgcn_readlane((uint32_t)(key >> 32), k);
        const uint64_t other = (uint64_t)hi << 32 | lo;
        rank += other > key || (other == key && k < t); // groups without elements have equal keys
      }
      if (rank == out.top_n - 1) bound_key = key;
    }
    __syncthreads();
    const uint64_t bound = bound_key;
    if (mine && mine >= bound) {
      for (int k = t; k * kV < vocab; k += kThreads) {
#pragma unroll
        for (int e = 0; e < kV; ++e) {
          if (k * kV + e >= vocab) break;
          const float x = (float)row[k * kV + e];
          if (key_of(x, k) >= bound) {
            const uint32_t at = atomicAdd(&n_found, 1u);
            if (at < kCandidates) found[at] = key_of(x, k * kV + e);
          }
        }
      }
    }
    __syncthreads();
    const uint32_t n = n_found;
    if (n > kCandidates) return find_by_rounds<T, kThreads>(row, vocab, out.top_n, logprob_of, ids, values, keys);
    for (uint32_t k = t; k < n; k += kThreads) { // ranked by counting: all keys differ
      const uint64_t key = found[k];
      int rank = 0;
      for (uint32_t j = 0; j < n; ++j) rank += found[j] > key;
      if (rank < out.top_n) {
        if (ids) ids[rank] = 0xFFFFFFFFu - (uint32_t)key;
        if (values) values[rank] = logprob_of(value_of(key >> 32));
      }
    }
  }
}

constexpr int kBackThreads = 256;
constexpr int kBackVectors = 4; // a lane's vectors, about

// A workgroup takes one of `segments` pieces of a row.
template <typename T> __global__ __launch_bounds__(kBackThreads) void token_logprobs_back(Logits in, hf_logprobs_grad g, uint32_t segments, uint32_t per_segment) {
  constexpr int kV = kVec<T>;
  typedef typename Vector<T>::type V;
  const int64_t r = blockIdx.x / segments;
  const int vocab = in.vocab, n_vec = vocab / kV;
  const int begin = blockIdx.x % segments * per_segment, end = min(begin + (int)per_segment, n_vec);
  const bool last = begin <= n_vec && n_vec < begin + (int)per_segment; // the piece with the elements past the whole vectors
  const int64_t target = target_of(in, r);
  T *to = static_cast<T *>(g.dlogits) + r * g.dlogits_stride;
  if (target < 0 || target >= vocab) {
    for (int i = begin + threadIdx.x; i < end; i += kBackThreads) *reinterpret_cast<typename Vector<T>::any *>(to + (int64_t)i * kV) = V{};
    if (last && (int)threadIdx.x < vocab - n_vec * kV) to[n_vec * kV + threadIdx.x] = (T)0.f;
    return;
  }
  const T *row = static_cast<const T *>(in.data) + r * in.row_stride;
  const float x_max = g.norm[2 * r], log_z = g.norm[2 * r + 1], gp = g.grad_logprob ? g.grad_logprob[r] : 0.f, gh = g.grad_entropy ? g.grad_entropy[r] : 0.f;
  const float ent = g.grad_entropy ? g.entropy[r] : 0.f, inv_t = in.inv_temperature;
  const float from = x_max == -INFINITY ? 0.f : x_max, less = log_z == -INFINITY ? 0.f : log_z; // a row of -inf: p = 0
  const float at0 = -inv_t * fmaf(gh, ent, gp), at1 = -inv_t * gh, hot = inv_t * gp;
  const auto grad = [&](float x, int j) {
    const float logp = fmaf(x - from, inv_t, -less);
    const float p = __builtin_amdgcn_exp2f(logp * kLog2e);
    float d = p * fmaf(at1, fmaxf(logp, -200.f), at0);
    return j == target ? d + hot : d;
  };
  for (int i = begin + threadIdx.x; i < end; i += kBackThreads) {
    const V v = load_vec(row + (int64_t)i * kV);
    V d;
#pragma unroll
    for (int e = 0; e < kV; ++e) d[e] = (T)grad((float)v[e], i * kV + e);
    *reinterpret_cast<typename Vector<T>::any *>(to + (int64_t)i * kV) = d;
  }
  if (last && (int)threadIdx.x < vocab - n_vec * kV) {
    const int j = n_vec * kV + threadIdx.x;
    to[j] = (T)grad((float)row[j], j);
  }
}

Logits logits_of(const hf_logits &in) { return {in.logits, in.targets, in.row_stride, in.vocab, in.target_bytes, in.inv_temperature}; }

template <typename T, int kThreads> hipError_t launch_threads(const hf_logits &in, const hf_logprobs &out, hipStream_t st) {
  const dim3 grid((uint32_t)in.rows);
  if (out.top_n) return enqueue_kernel(token_logprobs<T, kThreads, true>, grid, kThreads, st, logits_of(in), out);
  return enqueue_kernel(token_logprobs<T, kThreads, false>, grid, kThreads, st, logits_of(in), out);
}
template <typename T> hipError_t launch(const hf_logits &in, const hf_logprobs &out, hipStream_t st) {
  const int n_vec = in.vocab / kVec<T>;
  if (n_vec <= 512) return launch_threads<T, 64>(in, out, st);
  if (n_vec <= 8192) return launch_threads<T, 256>(in, out, st);
  return launch_threads<T, 1024>(in, out, st);
}

int vec_of(int dtype) { return dtype == HF_F32 ? kVec<float> : kVec<__bf16>; }

} // namespace

uint32_t logprob_back_segments(const hf_logits &in) {
  const uint32_t vectors = in.vocab / vec_of(in.dtype) + 1, per_wg = kBackThreads * kBackVectors;
  return (vectors + per_wg - 1) / per_wg;
}

int launch_token_logprobs(const hf_logits &in, const hf_logprobs &out, void *stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  return (int)(in.dtype == HF_BF16 ? launch<__bf16>(in, out, st) : in.dtype == HF_F16 ? launch<_Float16>(in, out, st) : launch<float>(in, out, st));
}

int launch_token_logprobs_back(const hf_logits &in, const hf_logprobs_grad &g, void *stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const uint32_t segments = logprob_back_segments(in), vectors = in.vocab / vec_of(in.dtype) + 1, per = (vectors + segments - 1) / segments;
  const dim3 grid((uint32_t)(in.rows * segments));
  const auto kernel = in.dtype == HF_BF16 ? token_logprobs_back<__bf16> : in.dtype == HF_F16 ? token_logprobs_back<_Float16> : token_logprobs_back<float>;
  return (int)enqueue_kernel(kernel, grid, kBackThreads, st, logits_of(in), g, segments, per);
}

} // namespace hf
