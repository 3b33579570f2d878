// Log probabilities of given tokens, the entropy and the likeliest tokens of rows of logits, and the gradient of the first two.
//
//   y = x / temperature;  m = max y;  z = sum e^(y-m);  lse = m + ln z;  logprob = y_t - lse;  H = ln z - sum e^(y-m) (y-m) / z
//   dx_j = ([j = t] g - p_j (g + h (ln p_j + H))) / temperature
//
// The forward pass reads every logit once and writes a few numbers a row; the gradient reads and writes each once.  HBM is
// the bound of the gradient (6.2 TB/s at 4096 x 32000 bf16, read and written) and of 32-bit logits (5.6 TB/s at 2048 x 128256).  At 2 bytes an element the forward pass has
// room for eleven vector operations on each and needs nine and a half (a base-2 exponential counts as four): 4.8 TB/s at 4096 x 32000, where vector instructions issue 71 % of
// the time.  A workgroup takes a row; every lane keeps its own running maximum, sum and weighted sum over its vectors and
// they are merged once at the end.
//
// The likeliest tokens come out of the same pass: besides its maximum a lane remembers in which of its vectors it first met it.
// The top_n-th largest of 64 groups' maxima bounds the top_n-th largest element from below, so only lanes whose own maximum reaches that
// bound can hold an answer; they, about top_n of them, read their vectors again (from L2, of long rows from beyond it: 1226 MB are
// fetched for the 1051 of 2048 x 128256 f32 with twenty tokens) and hand over what reaches the bound.  Keys are value and
// position together, so they are all different and ties fall to the lower id by themselves.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>

#include "lanes.hpp"
#include "logit_rows.hpp"
#include "rollout_kernels.hpp"

namespace hf {

namespace {

constexpr int kWave = 64;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kCandidates = 1024; // room for what reaches the bound; more go through find_by_rounds

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
  bool once; // more bytes than the memory-side cache could keep for a gradient that follows
};

__device__ __forceinline__ int64_t target_of(const Logits &in, int64_t row) {
  return in.target_bytes == 8 ? static_cast<const int64_t *>(in.targets)[row] : static_cast<const int32_t *>(in.targets)[row];
}

// Largest element m, and sums over the elements of 2^d and of 2^d d with d = (x - r) c - k, c = log2(e) / temperature.  Up to kWhole r is 0 and k the base x0 c
// rounded to a whole number: then d is one operation, with one rounding, and sums move to another k exactly, where x0 c itself would be off by as
// much as its own rounding.  Past it (mask values, low temperatures) that rounding alone would be a whole number and more: there r is x0 and k is 0.  x0 is
// the largest element of a lane's first vectors and follows m only when that is past it by kSlack of base 2, which for most lanes never happens.
struct Stats {
  float m, r, k, s, u;
};
constexpr float kSlack = 8, kWhole = 1 << 24;
__device__ __forceinline__ void rebase(Stats &st, float x0, float c) {
  const bool whole = fabsf(x0 * c) < kWhole;
  const float k = whole ? rintf(x0 * c) : 0.f, r = whole || x0 == -INFINITY ? 0.f : x0;
  const float d = st.s == 0 ? 0.f : fmaf(st.r - r, c, st.k - k); // (nothing to move before the first element)
  const float down = __builtin_amdgcn_exp2f(d);
  st.u = st.s > 0 ? down * fmaf(fmaxf(d, -200.f), st.s, st.u) : st.u;
  st.s *= down;
  st.r = r;
  st.k = k;
}
__device__ __forceinline__ Stats merge_wave(Stats st, float c) {
  st.m = over_wave<Max>(st.m);
  rebase(st, st.m, c);
  return {st.m, st.r, st.k, over_wave<Sum>(st.s), over_wave<Sum>(st.u)};
}

// limit: x0 and the slack
template <int kN> __device__ __forceinline__ void join(Stats &st, float &limit, const float (&x)[kN], float top, float c) {
  st.m = larger(st.m, top);
  if (top > limit) {
    rebase(st, top, c);
    limit = top + kSlack / c;
  }
  const auto add = [&](float d) {
    const float e = __builtin_amdgcn_exp2f(d); // NaN comes through here
    st.s += e;
    st.u = fmaf(e, fmaxf(d, -200.f), st.u); // 0 * -inf would be NaN, and 2^-200 is 0
  };
  if (st.r == 0) {
#pragma unroll
    for (int i = 0; i < kN; ++i) add(fmaf(x[i], c, -st.k));
  } else {
#pragma unroll
    for (int i = 0; i < kN; ++i) add((x[i] - st.r) * c);
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
  constexpr int kWaves = kThreads / kWave, kV = kVec<T>, kBatch = 4; // vectors that a lane takes at a time
  typedef typename Vector<T>::type V;
  __shared__ Stats stats[kWaves];
  __shared__ uint64_t group[kTop ? kWave : 1], found[kTop ? kCandidates : 1], bound_key;
  __shared__ uint32_t rank_of[kTop ? kWave : 1], lanes[kTop ? kThreads : 1], n_lanes, n_found;
  const int64_t r = blockIdx.x;
  const int t = threadIdx.x, lane = t % kWave, wave = t / kWave, vocab = in.vocab;
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
  const float x_target = (float)row[target];
  const float c = fminf(in.inv_temperature * kLog2e, FLT_MAX); // (times a difference of 0 it has to be 0)
  const int n_vec = vocab / kV; // whole ones
  Stats st = {-INFINITY, 0, 0, 0, 0};
  float limit = -INFINITY;
  float best = -INFINITY;         // the lane's largest element
  uint32_t best_at = 0xFFFFFFFFu; // and the vector that had it first; none: no vectors
  if constexpr (kTop) {
    if (t < kWave) group[t] = 0, rank_of[t] = 0;
    if (t == 0) n_lanes = n_found = 0;
    __syncthreads();
  }
  // kN vectors, kThreads apart from vector `at` on
  const auto add = [&](const auto &v, int at) {
    constexpr int kN = sizeof(v) / sizeof(v[0]);
    float x[kN * kV], tops[kN], top;
#pragma unroll
    for (int k = 0; k < kN; ++k) {
#pragma unroll
      for (int e = 0; e < kV; ++e) x[k * kV + e] = (float)v[k][e];
      tops[k] = larger(x[k * kV], x[k * kV + 1]);
#pragma unroll
      for (int e = 2; e < kV; e += 2) tops[k] = larger(tops[k], x[k * kV + e], x[k * kV + e + 1]);
      top = k ? larger(top, tops[k]) : tops[k];
    }
    if constexpr (kTop)
      if (top > best || best_at == 0xFFFFFFFFu) {
        best = top;
        best_at = at;
#pragma unroll
        for (int k = kN - 1; k > 0; --k)
          if (tops[k] == top) best_at = at + k * kThreads;
        if (tops[0] == top) best_at = at;
      }
    join(st, limit, x, top, c);
  };
  // the next vectors are on their way while the present ones are added
  int i = t;
  if (i + (kBatch - 1) * kThreads < n_vec) {
    V v[kBatch], next[kBatch];
    const auto load_batch = [&](V(&to)[kBatch], int at) {
      if (in.once) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) to[k] = load_once(row + (int64_t)(at + k * kThreads) * kV);
      } else {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) to[k] = load_vec(row + (int64_t)(at + k * kThreads) * kV);
      }
    };
    load_batch(v, i);
    // (no branch around the loads: the compiler could not tell how many are on their way, and would wait for all)
    for (; i + (2 * kBatch - 1) * kThreads < n_vec; i += kBatch * kThreads) {
      load_batch(next, i + kBatch * kThreads);
      add(v, i);
      for (int k = 0; k < kBatch; ++k) v[k] = next[k];
    }
    add(v, i);
    i += kBatch * kThreads;
  }
  { // fewer than kBatch are left, and the vector that the row ends in
    V v[kBatch - 1];
#pragma unroll
    for (int k = 0; k < kBatch - 1; ++k)
      if (i + k * kThreads < n_vec) v[k] = load_vec(row + (int64_t)(i + k * kThreads) * kV);
#pragma unroll
    for (int k = 0; k < kBatch - 1; ++k)
      if (i + k * kThreads < n_vec) {
        const V one[1] = {v[k]};
        add(one, i + k * kThreads);
      }
  }
  if (n_vec % kThreads == t && n_vec * kV < vocab) {
    V last[1];
#pragma unroll
    for (int e = 0; e < kV; ++e) last[0][e] = n_vec * kV + e < vocab ? row[n_vec * kV + e] : (T)-INFINITY;
    add(last, n_vec);
  }

  const uint64_t mine = kTop && best_at != 0xFFFFFFFFu ? key_of(best, best_at) : 0;
  if constexpr (kTop) atomicMax(reinterpret_cast<unsigned long long *>(&group[lane]), (unsigned long long)mine);
  st = merge_wave(st, c);
  if constexpr (kWaves > 1) {
    if (lane == 0) stats[wave] = st;
  }
  if constexpr (kWaves > 1 || kTop) __syncthreads();
  if constexpr (!kTop)
    if (wave > 0) return; // the rest is a few numbers
  if constexpr (kWaves > 1) st = merge_wave(lane < kWaves ? stats[lane] : Stats{-INFINITY, 0, 0, 0, 0}, c);
  // of base e: lse = top + log_z
  const float top = st.m == -INFINITY ? 0.f : st.m * in.inv_temperature, log2_s = __builtin_amdgcn_logf(st.s);
  const float past = st.m == -INFINITY ? 0.f : fmaf(st.m - st.r, c, -st.k), log_z = (log2_s - past) * kLn2;
  const auto logprob_of = [&](float x) { // nearer than x * inv_temperature - lse, whose terms are rounded where they are large
    return x == -INFINITY && st.s == st.s ? -INFINITY : (x - (st.m == -INFINITY ? 0.f : st.m)) * in.inv_temperature - log_z;
  };
  if (t == 0) {
    if (out.lse) out.lse[r] = top + log_z;
    if (out.norm) out.norm[2 * r] = st.m, out.norm[2 * r + 1] = log_z;
    if (out.entropy) out.entropy[r] = st.s == 0 ? 0.f : (log2_s - st.u / st.s) * kLn2;
    if (out.logprob) out.logprob[r] = logprob_of(x_target);
  }
  if constexpr (kTop) {
    int32_t *ids = out.top_ids ? out.top_ids + r * out.top_n : nullptr;
    float *values = out.top_logprobs ? out.top_logprobs + r * out.top_n : nullptr;
    { // the rank of every group's key; every wavefront counts a share of the others
      const uint64_t key = group[lane];
      uint32_t above = 0;
#pragma unroll
      for (int k = 0; k < kWave / kWaves; ++k) {
        const int j = wave * (kWave / kWaves) + k;
        const uint64_t other = group[j];
        above += other > key || (other == key && j < lane); // groups without elements have equal keys
      }
      atomicAdd(&rank_of[lane], above);
    }
    __syncthreads();
    if (t < kWave && rank_of[t] == (uint32_t)out.top_n - 1) bound_key = group[t];
    __syncthreads();
    const uint64_t bound = bound_key;
    if (mine && mine >= bound) lanes[atomicAdd(&n_lanes, 1u)] = t;
    __syncthreads();
    // the vectors of those lanes, dealt out over the workgroup
    const int each = (n_vec + (n_vec * kV < vocab) + kThreads - 1) / kThreads, n_pairs = n_lanes * each;
    for (int pair = t; pair < n_pairs; pair += kThreads) {
      const int k = lanes[pair / each] + pair % each * kThreads;
      V v;
      if (k < n_vec) {
        v = load_vec(row + (int64_t)k * kV);
      } else {
#pragma unroll
        for (int e = 0; e < kV; ++e) v[e] = (int64_t)k * kV + e < vocab ? row[(int64_t)k * kV + e] : (T)-INFINITY;
      }
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        const float x = (float)v[e];
        if (key_of(x, k) >= bound && (int64_t)k * kV + e < vocab) {
          const uint32_t at = atomicAdd(&n_found, 1u);
          if (at < kCandidates) found[at] = key_of(x, k * kV + e);
        }
      }
    }
    __syncthreads();
    const uint32_t n = n_found;
    // fewer than top_n: a signalling NaN was somebody's largest element
    if (n > kCandidates || n < (uint32_t)out.top_n) return find_by_rounds<T, kThreads>(row, vocab, out.top_n, logprob_of, ids, values, found);
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

// A workgroup takes one of `segments` pieces of a row.  Both sides are non-temporal: stored plainly, the gradient's lines have yet to be
// written to memory when the next forward pass reads (4096 x 32000 bf16, us, plain / non-temporal: this 72.7 / 70.6, the next forward 58 / 41).
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
    for (int i = begin + threadIdx.x; i < end; i += kBackThreads) store_once(to + (int64_t)i * kV, V{});
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
    const V v = load_once(row + (int64_t)i * kV);
    V d;
#pragma unroll
    for (int e = 0; e < kV; ++e) d[e] = (T)grad((float)v[e], i * kV + e);
    store_once(to + (int64_t)i * kV, d);
  }
  if (last && (int)threadIdx.x < vocab - n_vec * kV) {
    const int j = n_vec * kV + threadIdx.x;
    to[j] = (T)grad((float)row[j], j);
  }
}

// The forward pass reads plainly up to 512 MiB, so that the memory-side cache (256 MiB) keeps what it can for the gradient.  us, plain /
// non-temporal, when this was chosen: 4096 x 32000 bf16 forward then gradient 41 + 71 / 38 + 88 (forward alone 40 / 36), 2048 x 128256 f32 forward 188 / 183.
Logits logits_of(const hf_logits &in) {
  const bool once = in.rows * (int64_t)in.vocab * (in.dtype == HF_F32 ? 4 : 2) > (int64_t)512 << 20;
  return {in.logits, in.targets, in.row_stride, in.vocab, in.target_bytes, in.inv_temperature, once};
}

template <typename T, int kThreads> hipError_t launch_threads(const hf_logits &in, const hf_logprobs &out, hipStream_t st) {
  const dim3 grid((uint32_t)in.rows);
  if (out.top_n) return enqueue_kernel(token_logprobs<T, kThreads, true>, grid, kThreads, st, logits_of(in), out);
  return enqueue_kernel(token_logprobs<T, kThreads, false>, grid, kThreads, st, logits_of(in), out);
}
template <typename T> hipError_t launch(const hf_logits &in, const hf_logprobs &out, hipStream_t st) {
  // Lanes for a row, by its vectors: few rows in flight at a time are better for memory, but a lane wants a few vectors (what a wavefront does once a row is worth 40
  // elements a lane).  us at 64 / 256 / 512 / 1024 lanes: 1361 x 5004 f16 (625 vectors) 7.6 / 7.0 / 7.8 / 11.3, 64 x 32000 bf16 with alternatives (4000) 20.7 / 8.9 / 8.5 /
  // 8.9, 4096 x 32000 42 / 38 / 36 / 47, 2048 x 128256 f32 with alternatives (32064) 546 / 256 / 218 / 187.
  const int n_vec = in.vocab / kVec<T>;
  if (n_vec <= 512) return launch_threads<T, 64>(in, out, st);
  if (n_vec <= 2048) return launch_threads<T, 256>(in, out, st);
  if (n_vec <= 8192) return launch_threads<T, 512>(in, out, st);
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
