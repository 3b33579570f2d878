// Distillation from a teacher's top tokens: the divergence of rows of logits from it, and the gradient.
//
// Named tokens j with teacher's q_j and student's p_j = softmax(x / T)_j, and the rest as one more (or left out):
//   ahead = sum q (ln q - ln p),  back = sum p (ln p - ln q),  loss = (1 - w) ahead + w back
//   T dloss/dx_j = (1 - w) (p_j Q - q_j) + w p_j (ln p_j - ln q_j + 1 - back - P)      Q = sum q, P = sum p over what is counted
//   and of a token i that is not named the same with its rest's numbers, times its share of it:
//   T dloss/dx_i = e^(x_i / T) / sum of the others' e^(x / T) * ((1 - w) (p_rest Q - q_rest) + w p_rest (ln p_rest - ln q_rest + 1 - back - P))
//
// The forward pass reads every logit once and sums the exponentials of those that are not named: what is left of 1 beside a few likely tokens would be lost in a
// difference of two sums.  Which are named stands in a bitmap in shared memory, a byte to a vector of 8.  The named tokens are a few numbers a row, taken in 64 bits
// (a difference of logarithms near 1, one minus a sum of probabilities).  The gradient reads and writes every logit once; its named elements come out of a list.
//
// HBM is the bound of both where rows are many and long: forward 160 us (6.6 TB/s) and gradient 333 us (6.3 TB/s) of 2048 x 128256 f32, 44 and 61 us of 4096 x 32000 bf16 with a third of the rows left
// out (4.0 and, partly from the memory-side cache, 7.2).  Short rows and few are bound by what follows one another: the list, the bitmap, the logits, joining wavefronts, and some twenty operations of
// 64 bits on a chain (10 us forward for 1361 x 5004 f16, 7.4 for 64 x 32000 bf16).  Asking for the logits only when the list was known, and all wavefronts at the end, took 94 us for the 44.
#include <hip/hip_runtime.h>

#include <cfloat>

#include "lanes.hpp"
#include "logit_rows.hpp"
#include "step_kernels.hpp"

namespace hf {

namespace {

constexpr int kWave = 64;
constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;
// tokens that the bitmap spans at a time: every row that has so few lanes, or as many as 16 KiB hold
constexpr int window_of(int threads) { return threads == 64 ? 1 << 13 : threads == 256 ? 1 << 15 : 1 << 17; }

struct Logits {
  const void *data;
  int64_t row_stride;
  int32_t vocab;
  float inv_temperature;
};

// Largest element m, and the sum over the elements of 2^d with d = (x - r) c - k, c = log2(e) / temperature.  r and k follow the first elements and then only
// what is past them by kSlack of base 2; below kWhole r is 0 and k a whole number, so that d is one operation and sums move to another k exactly.
struct Stats {
  float m, r, k, s;
};
constexpr float kSlack = 8, kWhole = 1 << 24;
__device__ __forceinline__ void rebase(Stats &st, float x0, float c) {
  const bool whole = fabsf(x0 * c) < kWhole;
  const float k = whole ? rintf(x0 * c) : 0.f, r = whole || x0 == -INFINITY ? 0.f : x0;
  const float d = st.s == 0 ? 0.f : fmaf(st.r - r, c, st.k - k); // (nothing to move before the first element)
  st.s *= __builtin_amdgcn_exp2f(d);
  st.r = r;
  st.k = k;
}
__device__ __forceinline__ Stats merge_wave(Stats st, float c) {
  st.m = over_wave<Max>(st.m);
  rebase(st, st.m, c);
  return {st.m, st.r, st.k, over_wave<Sum>(st.s)};
}
template <int kN> __device__ __forceinline__ void join(Stats &st, float &limit, const float (&x)[kN], float c) {
  float top = larger(x[0], x[1]);
#pragma unroll
  for (int i = 2; i < kN; i += 2) top = larger(top, x[i], x[i + 1]);
  st.m = larger(st.m, top);
  if (top > limit) {
    rebase(st, top, c);
    limit = top + kSlack / c;
  }
  if (st.r == 0) {
#pragma unroll
    for (int i = 0; i < kN; ++i) st.s += __builtin_amdgcn_exp2f(fmaf(x[i], c, -st.k)); // NaN comes through here
  } else {
#pragma unroll
    for (int i = 0; i < kN; ++i) st.s += __builtin_amdgcn_exp2f((x[i] - st.r) * c);
  }
}

// over the wavefront, in registers
__device__ __forceinline__ double sum_wave(double x) {
  const auto halves = [](double y, float &lo, float &hi) { lo = __builtin_bit_cast(float, __double2loint(y)), hi = __builtin_bit_cast(float, __double2hiint(y)); };
  const auto whole = [](float lo, float hi) { return __hiloint2double(__builtin_bit_cast(int, hi), __builtin_bit_cast(int, lo)); };
  float lo, hi;
  halves(x, lo, hi), x += whole(dpp<0xB1>(lo), dpp<0xB1>(hi));
  halves(x, lo, hi), x += whole(dpp<0x4E>(lo), dpp<0x4E>(hi));
  halves(x, lo, hi), x += whole(dpp<0x141>(lo), dpp<0x141>(hi));
  halves(x, lo, hi), x += whole(dpp<0x140>(lo), dpp<0x140>(hi));
  float lo2, hi2;
  halves(x, lo, hi), lo2 = lo, hi2 = hi;
  swap32(lo, lo2), swap32(hi, hi2);
  x = whole(lo, hi) + whole(lo2, hi2);
  halves(x, lo, hi), lo2 = lo, hi2 = hi;
  swap16(lo, lo2), swap16(hi, hi2);
  return whole(lo, hi) + whole(lo2, hi2);
}

// kPlaces: of the list, to a lane of the wavefront that finishes a row; kOnce: past the caches
template <typename T, int kThreads, int kPlaces, bool kOnce> __global__ __launch_bounds__(kThreads) void top_distill(Logits in, hf_distillation a) {
  constexpr int kWaves = kThreads / kWave, kV = kVec<T>, kBatch = sizeof(T) == 4 ? 4 : 2, kWindow = window_of(kThreads);
  typedef typename Vector<T>::type V;
  __shared__ uint32_t named[kWindow / 32];
  __shared__ int32_t ids[kPlaces * kWave], given[kPlaces * kWave]; // with a log probability; or without one
  __shared__ float log_q[kPlaces * kWave], x_of[kPlaces * kWave];
  __shared__ Stats stats[kWaves];
  __shared__ uint32_t any, twice;
  const int64_t r = blockIdx.x;
  const int t = threadIdx.x, lane = t % kWave, wave = t / kWave, vocab = in.vocab;
  const T *row = static_cast<const T *>(in.data) + r * in.row_stride;
  const float c = fminf(in.inv_temperature * kLog2e, FLT_MAX); // (times a difference of 0 it has to be 0)

  int32_t id = -1;
  float lq = 0;
  if (t < a.n) id = a.ids[r * a.n + t], lq = a.logprobs[r * a.n + t];
  // the first vectors are on their way while the list is looked over, and then the next ones while the present ones are added
  V v[kBatch];
  const auto load_batch = [&](V(&to)[kBatch], const T *from) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) to[k] = kOnce ? load_once(from + (int64_t)k * kThreads * kV) : load_vec(from + (int64_t)k * kThreads * kV);
  };
  const auto whole_batch = [&](int i, int n_vec) { return i + (kBatch - 1) * kThreads < n_vec; };
  if (whole_batch(t, min(kWindow, vocab) / kV)) load_batch(v, row + t * kV);

  if (t == 0) any = twice = 0;
  for (int i = t; i < (min(kWindow, vocab) + 31) / 32; i += kThreads) named[i] = 0;
  __syncthreads();
  for (int j = t; j < a.n; j += kThreads) {
    if (j != t) id = a.ids[r * a.n + j], lq = a.logprobs[r * a.n + j];
    const bool is = id >= 0 && id < vocab, names = is && lq != -INFINITY;
    given[j] = is ? id : -1, ids[j] = names ? id : -1, log_q[j] = lq;
    x_of[j] = is ? (float)row[id] : -INFINITY;
    if (names) any = 1;
  }
  __syncthreads();
  if (!any) {
    if (t == 0) {
      if (a.loss) a.loss[r] = 0;
      if (a.norm) a.norm[2 * r] = 0, a.norm[2 * r + 1] = INFINITY; // what the gradient knows such a row by
    }
    if (a.slopes)
      for (int j = t; j <= a.n; j += kThreads) a.slopes[r * (a.n + 1) + j] = 0;
    return;
  }

  Stats st = {-INFINITY, 0, 0, 0};
  float limit = -INFINITY;
  for (int window = 0; window < vocab; window += kWindow) {
    const int size = min(kWindow, vocab - window), n_vec = size / kV;
    const T *from = row + window;
    if (window) {
      __syncthreads();
      for (int i = t; i < (size + 31) / 32; i += kThreads) named[i] = 0;
      if (whole_batch(t, n_vec)) load_batch(v, from + t * kV);
      __syncthreads();
    }
    for (int j = t; j < a.n; j += kThreads)
      if (const int at = ids[j] - window; ids[j] >= 0 && at >= 0 && at < size)
        if (atomicOr(&named[at / 32], 1u << at % 32) >> at % 32 & 1) twice = 1;
    __syncthreads();
    const uint8_t *bytes = reinterpret_cast<const uint8_t *>(named);
    // kN vectors, kThreads apart from vector `at` on
    const auto add = [&](const auto &vectors, int at) {
      constexpr int kN = sizeof(vectors) / sizeof(vectors[0]);
      float x[kN * kV];
      uint32_t bits[kN];
#pragma unroll
      for (int k = 0; k < kN; ++k) {
        const int i = at + k * kThreads;
        bits[k] = kV == 8 ? bytes[i] : bytes[i / 2] >> (i % 2 * 4) & 15;
      }
#pragma unroll
      for (int k = 0; k < kN; ++k) {
#pragma unroll
        for (int e = 0; e < kV; ++e) x[k * kV + e] = (float)vectors[k][e];
        if (bits[k]) {
#pragma unroll
          for (int e = 0; e < kV; ++e) x[k * kV + e] = bits[k] >> e & 1 ? -INFINITY : x[k * kV + e];
        }
      }
      join(st, limit, x, c);
    };
    int i = t;
    if (whole_batch(i, n_vec)) {
      V next[kBatch];
      for (; whole_batch(i + kBatch * kThreads, n_vec); i += kBatch * kThreads) {
        load_batch(next, from + (int64_t)(i + kBatch * kThreads) * kV);
        add(v, i);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) v[k] = next[k];
      }
      add(v, i);
      i += kBatch * kThreads;
    }
    { // fewer than kBatch are left, and the vector that the row ends in
      V rest[kBatch - 1];
#pragma unroll
      for (int k = 0; k < kBatch - 1; ++k)
        if (i + k * kThreads < n_vec) rest[k] = load_vec(from + (int64_t)(i + k * kThreads) * kV);
#pragma unroll
      for (int k = 0; k < kBatch - 1; ++k)
        if (i + k * kThreads < n_vec) {
          const V one[1] = {rest[k]};
          add(one, i + k * kThreads);
        }
    }
    if (n_vec % kThreads == t && n_vec * kV < size) {
      V last[1];
#pragma unroll
      for (int e = 0; e < kV; ++e) last[0][e] = n_vec * kV + e < size ? from[n_vec * kV + e] : (T)-INFINITY;
      add(last, n_vec);
    }
  }
  st = merge_wave(st, c);
  if constexpr (kWaves > 1) {
    if (lane == 0) stats[wave] = st;
    __syncthreads();
    if (wave > 0) return; // the rest is a few numbers
    st = merge_wave(lane < kWaves ? stats[lane] : Stats{-INFINITY, 0, 0, 0}, c);
  } else {
    __syncthreads();
  }

  // From here on one wavefront, base e, 64 bits, relative to the row's largest element.  Place j of the list counts if it is the first that names its token.
  int lead[kPlaces]; // the place that stands for this one's token; -1: none
  float x_named[kPlaces], top = st.m;
  double q_[kPlaces], e_[kPlaces];
  const auto leads = [&](int k) { return lead[k] == lane + k * kWave; };
#pragma unroll
  for (int k = 0; k < kPlaces; ++k) {
    lead[k] = -1;
    const int j = lane + k * kWave;
    if (j >= a.n) continue;
    x_named[k] = x_of[j];
    if (ids[j] >= 0) lead[k] = j;
    if (given[j] >= 0 && (twice || ids[j] < 0)) // (a place without a log probability may hold a token that another one names)
      for (int i = a.n - 1; i >= 0; --i)
        if (ids[i] == given[j]) lead[k] = i;
    if (leads(k)) top = fmaxf(top, x_named[k]);
  }
  top = over_wave<Max>(top);
  const double inv_t = in.inv_temperature, w = a.reverse;
  const bool others = !(st.s <= 0), rest = others && a.flags & HF_DISTILL_REST;
  // ln of the others' sum, relative to their own largest and to the row's
  const double log_own = others ? log((double)st.s) + ((double)st.k - ((double)st.m - st.r) * c) * kLn2 : -INFINITY;
  const double log_others = others ? log_own + ((double)st.m - top) * inv_t : -INFINITY;
  const auto y_of = [&](int k) { return x_named[k] == -INFINITY ? -(double)INFINITY : ((double)x_named[k] - top) * inv_t; };
  double z = 0, q_sum = 0;
#pragma unroll
  for (int k = 0; k < kPlaces; ++k)
    if (leads(k)) {
      e_[k] = exp(y_of(k)), q_[k] = exp((double)log_q[lane + k * kWave]);
      z += e_[k], q_sum += q_[k];
    }
  const double e_others = exp(log_others);
  z = sum_wave(z) + e_others;
  q_sum = sum_wave(q_sum);
  const double log_z = log(z), scale = z == 0 ? 0 : 1 / z; // (a row of -inf: p = 0)
  const auto lp_of = [&](int k) { return x_named[k] == -INFINITY && z == z ? -(double)INFINITY : y_of(k) - log_z; };
  const double lp_others = others ? log_others - log_z : -INFINITY, p_others = e_others * scale;
  const double q_rest = rest ? fmax(1 - q_sum, 0.) : 0., p_rest = rest ? p_others : 0.;
  const double lq_rest = rest ? log(fmax(1 - q_sum, 0x1p-24)) : 0;
  double ahead = 0, back = 0, p_sum = 0;
#pragma unroll
  for (int k = 0; k < kPlaces; ++k)
    if (leads(k)) {
      const double l = log_q[lane + k * kWave], lp = lp_of(k), p = e_[k] * scale;
      if (q_[k] != 0) ahead += q_[k] * (l - lp);
      if (p != 0 || l != l) back += p * (lp - l);
      p_sum += p;
    }
  ahead = sum_wave(ahead);
  back = sum_wave(back);
  p_sum = sum_wave(p_sum) + p_rest;
  if (rest) {
    if (q_rest != 0) ahead += q_rest * ((q_rest < 0x1p-24 ? log(q_rest) : lq_rest) - lp_others);
    if (p_rest != 0) back += p_rest * (lp_others - lq_rest);
  }
  const double mass = q_sum + q_rest;
  if (lane == 0) {
    // (a direction without weight has no part, inf though it may be)
    if (a.loss) a.loss[r] = (float)((w < 1 ? (1 - w) * ahead : 0.) + (w > 0 ? w * back : 0.));
    if (a.norm) a.norm[2 * r] = st.m, a.norm[2 * r + 1] = (float)log_own;
  }
  if (!a.slopes) return;
  const auto slope = [&](double p, double q, double lp, double l) {
    return inv_t * ((w < 1 ? (1 - w) * (p * mass - q) : 0.) + (w > 0 && p != 0 ? w * p * (lp - l + 1 - back - p_sum) : 0.));
  };
  // what an unnamed token's share is multiplied by; without a rest its terms have no part
  const double other = rest ? slope(p_others, q_rest, lp_others, lq_rest) : inv_t * p_others * ((w < 1 ? (1 - w) * mass : 0.) - (w > 0 ? w * (back + p_sum) : 0.));
  float *slopes = a.slopes + r * (a.n + 1);
  bool behind = false; // whether a place takes what another one has
#pragma unroll
  for (int k = 0; k < kPlaces; ++k) {
    const int j = lane + k * kWave;
    if (j >= a.n) continue;
    double mine = 0;
    if (leads(k)) mine = slope(e_[k] * scale, q_[k], lp_of(k), log_q[j]);
    else if (lead[k] >= 0) behind = true;
    else if (given[j] >= 0 && x_named[k] != -INFINITY) mine = other * exp(((double)x_named[k] - st.m) * inv_t - log_own); // one of the others
    x_of[j] = (float)mine;
    if (leads(k) || lead[k] < 0) slopes[j] = (float)mine;
  }
  if (lane == 0) slopes[a.n] = (float)other;
  if (__ballot(behind)) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < kPlaces; ++k)
      if (lane + k * kWave < a.n && lead[k] >= 0 && !leads(k)) slopes[lane + k * kWave] = x_of[lead[k]];
  }
}

constexpr int kBackThreads = 256;
// A lane's vectors.  us at 1 / 2 / 4: 2048 x 128256 f32 383 / 348 / 387, 1361 x 5004 f32 14.0 / 11.6 / 13.7; of 16 bits two take 21 for the 16.5 of forward and gradient of 1361 x 5004.
template <typename T> constexpr int kBackVectors = sizeof(T) == 4 ? 2 : 4;

// A workgroup takes one of `segments` pieces of a row.  Both sides go past the caches: with plain stores (loads) 2048 x 128256 f32 forward and gradient take 564 (510) us for 493.
template <typename T> __global__ __launch_bounds__(kBackThreads) void top_distill_back(Logits in, hf_distillation_grad g, uint32_t segments) {
  constexpr int kV = kVec<T>, kVectors = kBackVectors<T>, kPiece = kBackThreads * kVectors * kV;
  typedef typename Vector<T>::type V;
  __shared__ uint32_t named[kPiece / 32];
  __shared__ T value[kPiece]; // of the named elements alone
  const int t = threadIdx.x;
  const int64_t r = blockIdx.x / segments;
  const int begin = blockIdx.x % segments * kPiece, size = min(kPiece, in.vocab - begin), n_vec = size / kV;
  T *to = static_cast<T *>(g.dlogits) + r * g.dlogits_stride + begin;
  const float m = g.norm[2 * r], log_sum = g.norm[2 * r + 1];
  if (log_sum == INFINITY) { // no named tokens
    for (int i = t; i < n_vec; i += kBackThreads) store_once(to + i * kV, V{});
    if (const int i = n_vec * kV + t; t < kV && i < size) to[i] = (T)0.f;
    return;
  }
  const T *row = static_cast<const T *>(in.data) + r * in.row_stride + begin;
  V v[kVectors];
#pragma unroll
  for (int k = 0; k < kVectors; ++k)
    if (t + k * kBackThreads < n_vec) v[k] = load_once(row + (t + k * kBackThreads) * kV);
  const float scale = g.grad_loss[r], *slopes = g.slopes + r * (g.n + 1);
  for (int i = t; i < kPiece / 32; i += kBackThreads) named[i] = 0;
  __syncthreads();
  for (int j = t; j < g.n; j += kBackThreads) {
    const int64_t at = (int64_t)g.ids[r * g.n + j] - begin;
    if (at < 0 || at >= size) continue;
    atomicOr(&named[at / 32], 1u << at % 32);
    value[at] = (T)(scale * slopes[j]); // where a token comes twice both places hold the same
  }
  __syncthreads();
  const float factor = scale * slopes[g.n], inv_t = in.inv_temperature;
  const float from = m == -INFINITY ? 0.f : m, less = log_sum == -INFINITY ? 0.f : log_sum; // nothing else has p > 0
  const auto grad = [&](float x) {
    return factor * __builtin_amdgcn_exp2f(fmaf(x - from, inv_t, -less) * kLog2e);
  };
  const uint8_t *bytes = reinterpret_cast<const uint8_t *>(named);
#pragma unroll
  for (int k = 0; k < kVectors; ++k) {
    const int i = t + k * kBackThreads;
    if (i >= n_vec) break;
    const uint32_t bits = kV == 8 ? bytes[i] : bytes[i / 2] >> (i % 2 * 4) & 15;
    V d;
#pragma unroll
    for (int e = 0; e < kV; ++e) d[e] = (T)grad((float)v[k][e]);
    if (bits) {
#pragma unroll
      for (int e = 0; e < kV; ++e)
        if (bits >> e & 1) d[e] = value[i * kV + e];
    }
    store_once(to + i * kV, d);
  }
  if (const int i = n_vec * kV + t; t < kV && i < size) to[i] = named[i / 32] >> i % 32 & 1 ? value[i] : (T)grad((float)row[i]);
}

Logits logits_of(const hf_logits &in) { return {in.logits, in.row_stride, in.vocab, in.inv_temperature}; }

// The forward pass reads plainly up to 512 MiB, so that the memory-side cache (256 MiB) keeps what it can for the gradient.  us, plain / non-temporal, forward and gradient of
// 4096 x 32000 bf16 118 / 134, of 2048 x 128256 f32 486 / 493, of 4096 x 128256 bf16 549 / 541; forward alone 178 / 163 and 184 / 171.  Rows in falling order for the gradient are level or up to 4 % behind.
template <typename T, int kThreads> hipError_t launch_threads(const hf_logits &in, const hf_distillation &a, hipStream_t st) {
  const dim3 grid((uint32_t)in.rows);
  const bool once = in.rows * (int64_t)in.vocab * (int64_t)sizeof(T) > (int64_t)512 << 20;
  constexpr int kMost = HF_MAX_DISTILL / kWave;
  const auto kernel = a.n <= kWave ? once ? top_distill<T, kThreads, 1, true> : top_distill<T, kThreads, 1, false>
                                   : once ? top_distill<T, kThreads, kMost, true> : top_distill<T, kThreads, kMost, false>;
  return enqueue_kernel(kernel, grid, kThreads, st, logits_of(in), a);
}
// Lanes for a row, by its vectors; a lane takes two at a time of 16-bit elements, four of 32-bit ones.  us at 256 / 512 / 1024 lanes: 1000 x 16000 bf16 (2000 vectors) 11.6 / 13.7 / 17.4, 2048 x 32000 bf16
// (4000) 30.0 / 28.0 / 37.7, 64 x 32000 8.4 / 7.5 / 7.4, 1024 x 32000 f32 (8000) 26.2 / 24.9 / 28.0, 64 x 128256 bf16 (16032) 18.3 / 12.8 / 11.8, 1024 x 128256 58.5 / 59.3 / 58.2; four at a time of 16 bits
// 38 for the 28, two of 32 bits 206 for 197 (2048 x 128256).
template <typename T> hipError_t launch(const hf_logits &in, const hf_distillation &a, hipStream_t st) {
  const int n_vec = in.vocab / kVec<T>;
  if (n_vec <= 512) return launch_threads<T, 64>(in, a, st);
  if (n_vec <= 2048) return launch_threads<T, 256>(in, a, st);
  if (n_vec <= 8192) return launch_threads<T, 512>(in, a, st);
  return launch_threads<T, 1024>(in, a, st);
}

} // namespace

uint32_t distill_back_segments(const hf_logits &in) {
  const uint32_t piece = kBackThreads * (in.dtype == HF_F32 ? kBackVectors<float> * kVec<float> : kBackVectors<__bf16> * kVec<__bf16>);
  return (in.vocab + piece - 1) / piece;
}

int launch_top_distill(const hf_logits &in, const hf_distillation &a, void *stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  return (int)(in.dtype == HF_BF16 ? launch<__bf16>(in, a, st) : in.dtype == HF_F16 ? launch<_Float16>(in, a, st) : launch<float>(in, a, st));
}

int launch_top_distill_back(const hf_logits &in, const hf_distillation_grad &g, void *stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const uint32_t segments = distill_back_segments(in);
  const dim3 grid((uint32_t)(in.rows * segments));
  const auto kernel = in.dtype == HF_BF16 ? top_distill_back<__bf16> : in.dtype == HF_F16 ? top_distill_back<_Float16> : top_distill_back<float>;
  return (int)enqueue_kernel(kernel, grid, kBackThreads, st, logits_of(in), g, segments);
}

} // namespace hf
