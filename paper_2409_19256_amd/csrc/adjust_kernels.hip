// Logits on their way to a choice of token: penalties for repeated tokens, biases, tokens that a grammar rules out.
//
//   seen: x > 0 ? x / r : x r;   n times in the answer: - f n - p;   bias: + b;   ruled out: -inf
//
// Every logit is read once and written once, so HBM is the bound.  A workgroup takes a piece of a row: it asks for its logits, counts the row's tokens that
// fall into the piece in shared memory while they are on their way, lays them there, changes those that were counted or have a bias, each by one lane (whose bias
// is the token's last, or who is first to take the count away), and writes the piece.  The work beside the copy goes by the tokens and biases, not by the logits: a look at
// every logit's count took more than HBM leaves room for.  In place, of rows without a mask and with few tokens, nothing is moved but what changes.
//
// us, out of place, beside the copy alone by the same workgroups: 1024 x 32000 bf16, 900 tokens a row, half of the rows masked 24.7 beside 22.5; 1024 x 128256 f32, 2800 tokens and 64 biases a row,
// half masked 194-208 beside 165-175 (5.1-5.4 TB/s); 64 x 32000 bf16 4.8, one workgroup after another's data (lengths, tokens, counts, logits).  Pieces of 4096 / 8192 / 16384 (256 / 512 / 1024 lanes)
// take 33 / 27 / 26 and 254 / 210 / 245, so do 512 lanes for 4096 (35, 250) or 1024 for 8192 (35, 221).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "logit_rows.hpp"
#include "step_kernels.hpp"

namespace hf {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 512, kWave = 64;
constexpr int kChunk = 8192; // logits of a piece
constexpr int kHeld = 8;     // of a row's tokens that a lane keeps in registers
static_assert((int64_t)kMaxAdjustList + kThreads <= (int64_t)INT32_MAX + 1, "a lane's place in a list, kThreads further at a time, stays in 32 bits");

struct Row { // what one row's elements are changed by
  float rep, freq, pres;
};
// n: times in the answer, and whether the token is there at all
__device__ __forceinline__ float penalised(float x, uint32_t n, bool seen, const Row &row) {
  if (seen) x = x > 0 ? x / row.rep : x * row.rep;
  return n ? x - row.freq * (float)n - row.pres : x;
}

// How often tokens of the piece stand in the row: a number each, whose highest bit says that the token stands in the prompt.  16 bits are enough for
// rows of fewer than 2^15 tokens, two numbers to a word; others take a word each.
template <bool kWide> struct Counts {
  static constexpr int kWords = kWide ? kChunk : kChunk / 2;
  static constexpr uint32_t kPrompt = kWide ? 0x80000000u : 0x8000u;
  static __device__ __forceinline__ void add(uint32_t *words, int at, bool prompt) {
    const int shift = kWide ? 0 : at % 2 * 16;
    uint32_t *word = words + (kWide ? at : at / 2);
    if (prompt) atomicOr(word, kPrompt << shift);
    else atomicAdd(word, 1u << shift);
  }
  // the number, which is 0 for whoever asks next
  static __device__ __forceinline__ uint32_t take(uint32_t *words, int at) {
    if (kWide) return atomicExch(words + at, 0u);
    const int shift = at % 2 * 16;
    return atomicAnd(words + at / 2, ~(0xFFFFu << shift)) >> shift & 0xFFFFu;
  }
};

// the bits of vector `v` of a row: 8 elements or 4
template <typename T> __device__ __forceinline__ uint32_t bits_of(const uint8_t *allowed, int v) {
  return kVec<T> == 8 ? allowed[v] : allowed[v / 2] >> (v % 2 * 4) & 15u;
}

template <typename T, typename Token, bool kTables, bool kWide, bool kMany> __global__ __launch_bounds__(kThreads) void adjust_logits(hf_adjustment a, uint32_t pieces, int32_t few) {
  constexpr int kV = kVec<T>, kPer = kChunk / kV / kThreads; // vectors of a lane
  typedef typename Vector<T>::type V;
  typedef Counts<kWide> C;
  __shared__ __attribute__((aligned(16))) uint32_t count[kTables ? C::kWords : 1];
  __shared__ __attribute__((aligned(16))) T tile[kTables ? kChunk : 1];
  __shared__ __attribute__((aligned(16))) uint32_t last[kMany ? kChunk : 1]; // of the token's biases, its place in the list + 1
  const int t = threadIdx.x;
  // the pieces of a row on one XCD (workgroups go round them by eights), whose L2 then reads the row's tokens once: 1024 x 32000 bf16 24.2 us for 27.7
  const uint32_t turned = (uint32_t)(a.rows / 8) * 8 * pieces, b = blockIdx.x;
  const int64_t r = b < turned ? (int64_t)(b / 8 / pieces) * 8 + b % 8 : b / pieces;
  const int begin = (b < turned ? b / 8 % pieces : b % pieces) * kChunk, size = min(kChunk, a.vocab - begin), n_vec = size / kV; // whole vectors; the others are the row's last elements
  const T *from = static_cast<const T *>(a.logits) + r * a.row_stride + begin;
  T *to = static_cast<T *>(a.out) + r * a.out_stride + begin;
  const uint8_t *allowed = nullptr; // all
  if (a.allowed) {
    const int64_t g = a.allowed_rows ? a.allowed_rows[r] : r;
    if (g >= 0 && g < a.n_allowed) allowed = reinterpret_cast<const uint8_t *>(a.allowed + g * a.allowed_stride) + begin / 8;
  }
  const int n = kTables && a.tokens ? min(max(a.lens[r], 0), a.width) : 0;
  // In place, without a mask and with few tokens nothing is moved but what changes.
  const bool sparse = from == to && !allowed && n <= few;
  if (!kTables && sparse) return;
  const int n_last = sparse ? 0 : min(kV, size - n_vec * kV); // elements past the whole vectors, a lane each

  V v[kPer];
  uint32_t bits[kPer];
  if (!sparse) {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (t + k * kThreads < n_vec) v[k] = load_once(from + (t + k * kThreads) * kV);
    if (allowed) {
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (t + k * kThreads < n_vec) bits[k] = bits_of<T>(allowed, t + k * kThreads);
    }
  }
  if constexpr (kTables) {
    const int prompt = a.prompt_lens ? a.prompt_lens[r] : 0;
    const Row row = {a.repetition ? a.repetition[r] : 1.f, a.frequency ? a.frequency[r] : 0.f, a.presence ? a.presence[r] : 0.f};
    const Token *tokens = static_cast<const Token *>(a.tokens) + r * a.tokens_stride;
    Token held[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (t + k * kThreads < n) held[k] = tokens[t + k * kThreads];
    const int32_t *ids = a.bias_ids + r * a.n_bias;
    const int id = t < a.n_bias ? ids[t] : -1;
    const float bias = t < a.n_bias ? a.bias[r * a.n_bias + t] : 0.f;
    for (int i = t; i < C::kWords / 4; i += kThreads) reinterpret_cast<u32x4 *>(count)[i] = u32x4{0, 0, 0, 0};
    if constexpr (kMany)
      for (int i = t; i < kChunk / 4; i += kThreads) reinterpret_cast<u32x4 *>(last)[i] = u32x4{0, 0, 0, 0};
    __syncthreads();
    // f(place in the piece, place in the row) for the tokens of the piece
    const auto each = [&](const auto &f) {
#pragma unroll
      for (int k = 0; k < kHeld; ++k)
        if (t + k * kThreads < n)
          if (const int64_t at = (int64_t)held[k] - begin; at >= 0 && at < size) f((int)at, t + k * kThreads);
      for (int i = t + kHeld * kThreads; i < n; i += kThreads)
        if (const int64_t at = (int64_t)tokens[i] - begin; at >= 0 && at < size) f((int)at, i);
    };
    each([&](int at, int i) { C::add(count, at, i < prompt); });
    // f(place of the list, place in the piece, bias) for the biases of the piece
    const auto each_bias = [&](const auto &f) {
      if (id >= begin && id - begin < size) f(t, id - begin, bias);
      for (int j = t + kThreads; j < a.n_bias; j += kThreads)
        if (const int other = ids[j]; other >= begin && other - begin < size) f(j, other - begin, a.bias[r * a.n_bias + j]);
    };
    if constexpr (kMany) each_bias([&](int j, int at, float) { atomicMax(&last[at], j + 1u); });
    if (!sparse) {
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (t + k * kThreads < n_vec) *reinterpret_cast<V *>(tile + (t + k * kThreads) * kV) = v[k];
      if (t < n_last) tile[n_vec * kV + t] = from[n_vec * kV + t];
    }
    __syncthreads();
    const auto change = [&](int i, uint32_t counted, float add) {
      T *x = sparse ? to + i : tile + i;
      *x = (T)(penalised((float)*x, counted & ~C::kPrompt, counted != 0, row) + add);
    };
    if constexpr (kMany) {
      each_bias([&](int j, int at, float add) {
        if (last[at] == j + 1u) change(at, C::take(count, at), add);
      });
      __syncthreads();
    } else if (a.n_bias) {
      // up to 64 biases are in the first wavefront's lanes: those behind that are of the same token hold in place of theirs
      bool holds = id >= begin && id - begin < size;
      for (uint64_t left = t < kWave ? __ballot(holds) : 0; left; left &= left - 1) {
        const int l = __builtin_ctzll(left);
        if (__ballot(id == __builtin_amdgcn_readlane(id, l)) >> l > 1 && t == l) holds = false;
      }
      if (holds) change(id - begin, C::take(count, id - begin), bias);
      __syncthreads();
    }
    each([&](int at, int) {
      if (const uint32_t counted = C::take(count, at)) change(at, counted, 0.f);
    });
    if (sparse) return;
    __syncthreads();
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int at = t + k * kThreads;
    if (at >= n_vec) break;
    if constexpr (kTables) v[k] = *reinterpret_cast<const V *>(tile + at * kV);
    if (allowed) {
#pragma unroll
      for (int e = 0; e < kV; ++e) v[k][e] = bits[k] >> e & 1 ? v[k][e] : (T)-INFINITY;
    }
    store_once(to + at * kV, v[k]);
  }
  if (t < n_last) {
    const int i = n_vec * kV + t;
    const T x = kTables ? tile[i] : from[i];
    to[i] = !allowed || allowed[i / 8] >> i % 8 & 1 ? x : (T)-INFINITY;
  }
}

// More biases than lanes of a wavefront are settled in a table of the piece, which leaves room for two workgroups on a CU instead of three.  us, a lane to a bias / by the table: 64 biases in 1024 rows of
// 128256 f32 207 / 235, 16 in 64 rows of 32000 bf16 4.8 / 4.9.  Without the table (every bias against the others, 64 at a time): 300 in 4195 rows of 32000 f16 160 / 118, in 3 rows 8.7 / 4.7.
template <typename T, typename Token, bool kWide> hipError_t launch_tables(const hf_adjustment &a, const dim3 &grid, uint32_t pieces, int32_t few, hipStream_t st) {
  return enqueue_kernel(a.n_bias > kWave ? adjust_logits<T, Token, true, kWide, true> : adjust_logits<T, Token, true, kWide, false>, grid, kThreads, st, a, pieces, few);
}
// Tokens up to which a row in place and without a mask is changed in memory, each by itself, beside its biases: one costs what moving 36 bytes of the row does, and as much as 1/3800 of the
// row besides, since every piece goes through the whole list.  us, by the token / by the piece:
//   tokens                64           512          1024         1536         2048         2560         4096       few: up to
//   1024 x 32000 bf16   13.0 / 22.3  15.9 / 22.8  20.8 / 24.0  27.1 / 25.6  33.3 / 27.4  38.3 / 29.8  50.4 / 36.2     1230
//   64 x 32000 bf16      3.3 / 4.0    3.7 / 4.2    4.2 / 4.5    5.0 / 4.7    5.4 / 5.0    5.9 / 5.3    7.7 / 6.2      1230
//   4096 x 5004 f16     13.9 / 18.2  18.8 / 18.8  25.7 / 23.1  33.4 / 26.9  40.0 / 28.2  48.2 / 30.5  63.6 / 37.7      263
//   1024 x 32000 f32    13.8 / 44.4  18.2 / 46.4  26.6 / 45.8  35.4 / 47.3  43.8 / 47.9  50.9 / 49.9  68.4 / 54.0     1855
//   1024 x 128256 bf16  42.6 / 82.6  48.4 / 83.1  59.5 / 84.8  71.8 / 87.9  85.0 / 93.7  97.0 / 100    147 / 123      2490
//   1024 x 128256 f32   45.8 / 169   54.2 / 174   71.7 / 171   89.1 / 170    112 / 172    144 / 177    242 / 183      3000
template <typename T> int32_t few_tokens(const hf_adjustment &a) {
  const int64_t row = a.vocab * (int64_t)sizeof(T);
  return (int32_t)std::max<int64_t>(-1, row / (36 + row / 3800) - a.n_bias);
}
template <typename T> hipError_t launch(const hf_adjustment &a, hipStream_t st) {
  const uint32_t pieces = (a.vocab + kChunk - 1) / kChunk;
  const dim3 grid((uint32_t)(a.rows * pieces));
  const int32_t few = few_tokens<T>(a);
  const bool text = a.tokens && a.width, wide = text && a.width >= 1 << 15;
  if (text && a.token_bytes == 8) return wide ? launch_tables<T, int64_t, true>(a, grid, pieces, few, st) : launch_tables<T, int64_t, false>(a, grid, pieces, few, st);
  if (text || a.n_bias) return wide ? launch_tables<T, int32_t, true>(a, grid, pieces, few, st) : launch_tables<T, int32_t, false>(a, grid, pieces, few, st);
  if (a.logits == a.out && !a.allowed) return hipSuccess;
  return enqueue_kernel(adjust_logits<T, int32_t, false, false, false>, grid, kThreads, st, a, pieces, few);
}

} // namespace

bool adjust_fits(const hf_adjustment &a) {
  constexpr uint64_t kMost = kMaxLanes / kThreads; // workgroups
  return (uint64_t)a.rows <= kMost / ((a.vocab + kChunk - 1) / kChunk);
}

int launch_adjust(const hf_adjustment &a, void *stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  return (int)(a.dtype == HF_BF16 ? launch<__bf16>(a, st) : a.dtype == HF_F16 ? launch<_Float16>(a, st) : launch<float>(a, st));
}

} // namespace hf
