// Logits on their way to a choice of token: penalties for repeated tokens, biases, tokens that a grammar rules out.
//
//   seen: x > 0 ? x / r : x r;   n times in the answer: - f n - p;   bias: + b;   ruled out: -inf
//
// Every logit is read once and written once, so HBM is the bound.  A workgroup takes a piece of a row: it asks for its logits, counts the row's tokens that
// fall into the piece in shared memory while they are on their way, keeps them there, changes those that were counted or have a bias (each by one lane: the one that
// counted first, or whose bias is the last), and writes the piece.  In place nothing is moved but what changes.
#include <hip/hip_runtime.h>

#include "logit_rows.hpp"
#include "step_kernels.hpp"

namespace hf {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;                 // logits of a piece
constexpr uint32_t kPrompt = 0x80000000u;    // a count's bit: the token stands in the prompt

struct Row { // what one row's elements are changed by
  float rep, freq, pres;
  const float *bias;
  const uint8_t *allowed; // null: all
};

__device__ __forceinline__ float penalised(float x, uint32_t count, const Row &row) {
  if (count == 0) return x;
  x = x > 0 ? x / row.rep : x * row.rep;
  const uint32_t n = count & ~kPrompt;
  return n ? x - row.freq * (float)n - row.pres : x;
}

// the bits of vector `v` of a row: 8 elements or 4
template <typename T> __device__ __forceinline__ uint32_t allowed_of(const uint8_t *allowed, int v) {
  return kVec<T> == 8 ? allowed[v] : allowed[v / 2] >> (v % 2 * 4) & 15u;
}

template <typename T, bool kTables, bool kInPlace> __global__ __launch_bounds__(kThreads) void adjust_logits(hf_adjustment a, uint32_t pieces) {
  constexpr int kV = kVec<T>, kPer = kChunk / kV / kThreads; // vectors of a lane
  constexpr uint32_t kAll = (1u << kV) - 1;
  typedef typename Vector<T>::type V;
  __shared__ uint32_t count[kTables ? kChunk : 1], bias_at[kTables ? kChunk : 1];
  __shared__ __attribute__((aligned(16))) T tile[kTables && !kInPlace ? kChunk : 1];
  __shared__ uint16_t touched[kTables ? kChunk : 1];
  __shared__ uint32_t n_touched;
  const int t = threadIdx.x;
  const int64_t r = blockIdx.x / pieces;
  const int begin = blockIdx.x % pieces * kChunk, size = min(kChunk, a.vocab - begin), n_vec = size / kV; // whole vectors; the others are the row's last elements
  const T *from = static_cast<const T *>(a.logits) + r * a.row_stride + begin;
  T *to = static_cast<T *>(a.out) + r * a.out_stride + begin;
  Row row = {a.repetition ? a.repetition[r] : 1.f, a.frequency ? a.frequency[r] : 0.f, a.presence ? a.presence[r] : 0.f, nullptr, nullptr};
  if (a.n_bias) row.bias = a.bias + r * a.n_bias;
  if (a.allowed) {
    const int64_t g = a.allowed_rows ? a.allowed_rows[r] : r;
    if (g >= 0 && g < a.n_allowed) row.allowed = reinterpret_cast<const uint8_t *>(a.allowed + g * a.allowed_stride) + begin / 8;
  }
  const auto open = [&](int i) { return !row.allowed || row.allowed[i / 8] >> i % 8 & 1; };

  V v[kPer];
  if constexpr (!kInPlace) {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (t + k * kThreads < n_vec) v[k] = load_once(from + (t + k * kThreads) * kV);
  }
  if constexpr (kTables) {
    for (int i = t; i < kChunk; i += kThreads) count[i] = bias_at[i] = 0;
    if (t == 0) n_touched = 0;
    __syncthreads();
    if (a.tokens) {
      const int n = min(max(a.lens[r], 0), a.width), prompt = a.prompt_lens ? a.prompt_lens[r] : 0;
      const auto add = [&](int64_t token, int i) {
        const int64_t at = token - begin;
        if (at < 0 || at >= size) return;
        const uint32_t old = i < prompt ? atomicOr(&count[at], kPrompt) : atomicAdd(&count[at], 1u);
        if (old == 0) touched[atomicAdd(&n_touched, 1u)] = at;
      };
      if (a.token_bytes == 8) {
        const int64_t *tokens = static_cast<const int64_t *>(a.tokens) + r * a.tokens_stride;
        for (int i = t; i < n; i += kThreads) add(tokens[i], i);
      } else {
        const int32_t *tokens = static_cast<const int32_t *>(a.tokens) + r * a.tokens_stride;
        for (int i = t; i < n; i += kThreads) add(tokens[i], i);
      }
    }
    for (int j = t; j < a.n_bias; j += kThreads) {
      const int64_t at = (int64_t)a.bias_ids[r * a.n_bias + j] - begin;
      if (at >= 0 && at < size) atomicMax(&bias_at[at], j + 1u);
    }
    if constexpr (!kInPlace) {
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (t + k * kThreads < n_vec) *reinterpret_cast<V *>(tile + (t + k * kThreads) * kV) = v[k];
      if (const int i = n_vec * kV + t; t < kV && i < size) tile[i] = from[i];
    }
    __syncthreads();
    const auto change = [&](int i, float bias) {
      if constexpr (kInPlace) {
        if (open(i)) to[i] = (T)(penalised((float)to[i], count[i], row) + bias);
      } else {
        tile[i] = (T)(penalised((float)tile[i], count[i], row) + bias);
      }
    };
    for (uint32_t k = t; k < n_touched; k += kThreads)
      if (const int i = touched[k]; bias_at[i] == 0) change(i, 0.f);
    for (int j = t; j < a.n_bias; j += kThreads) {
      const int64_t at = (int64_t)a.bias_ids[r * a.n_bias + j] - begin;
      if (at >= 0 && at < size && bias_at[at] == j + 1u) change(at, row.bias[j]);
    }
    if constexpr (!kInPlace) __syncthreads();
  }
  if constexpr (kInPlace) {
    if (!row.allowed) return;
    for (int k = t; k < n_vec; k += kThreads) {
      const uint32_t bits = allowed_of<T>(row.allowed, k);
      if (bits == 0) {
        V ruled;
#pragma unroll
        for (int e = 0; e < kV; ++e) ruled[e] = (T)-INFINITY;
        *reinterpret_cast<typename Vector<T>::any *>(to + k * kV) = ruled;
      } else if (bits != kAll) {
#pragma unroll
        for (int e = 0; e < kV; ++e)
          if (!(bits >> e & 1)) to[k * kV + e] = (T)-INFINITY;
      }
    }
    if (const int i = n_vec * kV + t; t < kV && i < size && !open(i)) to[i] = (T)-INFINITY;
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int at = t + k * kThreads;
      if (at >= n_vec) break;
      if constexpr (kTables) v[k] = *reinterpret_cast<const V *>(tile + at * kV);
      if (row.allowed) {
        const uint32_t bits = allowed_of<T>(row.allowed, at);
#pragma unroll
        for (int e = 0; e < kV; ++e) v[k][e] = bits >> e & 1 ? v[k][e] : (T)-INFINITY;
      }
      *reinterpret_cast<typename Vector<T>::any *>(to + at * kV) = v[k];
    }
    if (const int i = n_vec * kV + t; t < kV && i < size) to[i] = open(i) ? (kTables ? tile[i] : from[i]) : (T)-INFINITY;
  }
}

template <typename T> hipError_t launch(const hf_adjustment &a, hipStream_t st) {
  const uint32_t pieces = (a.vocab + kChunk - 1) / kChunk;
  const dim3 grid((uint32_t)(a.rows * pieces));
  const bool tables = (a.tokens && a.width) || a.n_bias, in_place = a.logits == a.out;
  if (in_place && !tables && !a.allowed) return hipSuccess;
  const auto kernel = tables ? in_place ? adjust_logits<T, true, true> : adjust_logits<T, true, false> : in_place ? adjust_logits<T, false, true> : adjust_logits<T, false, false>;
  return enqueue_kernel(kernel, grid, kThreads, st, a, pieces);
}

} // namespace

uint64_t adjust_wgs(const hf_adjustment &a) { return (uint64_t)a.rows * ((a.vocab + kChunk - 1) / kChunk); }

int launch_adjust(const hf_adjustment &a, void *stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  return (int)(a.dtype == HF_BF16 ? launch<__bf16>(a, st) : a.dtype == HF_F16 ? launch<_Float16>(a, st) : launch<float>(a, st));
}

} // namespace hf
