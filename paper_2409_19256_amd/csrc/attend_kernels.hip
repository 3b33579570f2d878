// Attention of one query token per sequence over a paged cache, the samples of a prompt taking the prompt's pages together.
//
//   x_j = scale <q, k_j>,  m = max_j x_j,  l = sum_j exp(x_j - m),  o = sum_j exp(x_j - m) v_j / l
//
// Any cut of the tokens into parts gives (m, l, o) of each part, and parts merge exactly:
// m = max m_i, l = sum l_i exp(m_i - m), o likewise.  A prompt is cut into parts whose rows are all the queries of its samples that
// read one KV head (samples x query heads per KV head), a response into parts whose rows are the sequence's own query heads, and a
// second kernel merges a row's parts in a fixed order.  Short contexts are not cut: one workgroup takes prompt and response.
//
// Bound: a response's keys and values are read for one sequence alone, 4 bytes per (token, element) for 4 x rows operations, so
// HBM is the bound there; a prompt's for all of its samples' rows.  What keeps the loads wide and the wavefronts fed:
//  - a wavefront takes tiles of 32 tokens straight from memory into registers, keys and values of the next tile on their way while it works on
//    the present one; nothing is staged and no wavefront waits for another until its part is done.  Where a prompt has many
//    rows, eight wavefronts of a workgroup share its tokens and rows, so that a SIMD has two (prompts brought into LDS by the whole workgroup were
//    no faster: 54 us where this takes 51, 61 samples of 32749 tokens with 488 rows; a SIMD issues vector instructions 30 % of that time, its matrix unit
//    is busy 19 %, and two wavefronts hide no more of each other's waits);
//  - what is read for one workgroup alone goes past the caches (responses of the 7B shape, 1024 tokens each: 6.7 TB/s, plain loads 6.0);
//  - a page's number and address are the same for a whole wavefront and are worked out by the scalar unit (pages of 16 tokens and more);
//  - scores are made transposed, S^T = K Q^T: the accumulator then holds, for the query of a lane's column, four tokens of each 16, which
//    is what the second product O^T = V^T P^T wants as its right operand if its 32 tokens are taken in the order (16-token
//    half, lane group, token): P never moves between lanes;
//  - a lane loads 16 bytes of each of its eight tokens' values, whole rows over 16 lanes; the eight rows are turned in its registers (one byte
//    permute per two elements) into left operands for eight products, product j holding every eighth element of a head.
// Exponentials are of base 2, the scale carries the factor.  P is rounded to the cache's type twice, once for its upper bits and once for the
// rest: rounded once it would add as much to the error as the rounding of the output does.  Twice it is off by 2^-17 of itself in bfloat16; see kUp for float16.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "lanes.hpp"
#include "rollout_kernels.hpp"

namespace hf {

namespace {

constexpr int kThreads = 256, kWave = 64;
constexpr int kTile = 32;   // tokens of a tile
constexpr int kRowsTile = 16; // queries of a tile
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A: lane holds row lane % 16, k = 8 * (lane / 16) .. + 7; B: column lane % 16, the same k; C: column lane % 16, rows 4 * (lane / 16) .. + 3
template <typename T> struct Matrix;
template <> struct Matrix<__bf16> {
  typedef __bf16 Op __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 product(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Op, a), __builtin_bit_cast(Op, b), c, 0, 0, 0);
  }
};
template <> struct Matrix<_Float16> {
  typedef _Float16 Op __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 product(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Op, a), __builtin_bit_cast(Op, b), c, 0, 0, 0);
  }
};

struct AttendParams {
  hf_attention a;
  AttendShape s;
  const char *k, *v;
  int64_t page_bytes, head_bytes, token_bytes;
  uint32_t n_pages;
  int32_t n_kv_heads, head_dim, page_shift, ratio;
  float scale2;   // of base 2
  float *part_o;  // [row, part, head_dim]
  float *part_ml; // [row, part, 2]
};

// How heads are read: whole (head_dim is the kernel's), in pieces of 8 elements, or by single elements
enum { kWhole = 0, kPieces = 1, kElements = 2 };

// what is only read for the whole of a kernel, and from addresses that all lanes share, may come through the scalar cache
typedef const __attribute__((address_space(4))) int32_t *ScalarInts;
__device__ __forceinline__ int32_t load_scalar(const int32_t *p) { return *(ScalarInts)(uintptr_t)p; }

// single elements of a row, two to a register; zeros past the head
__device__ __forceinline__ uint32_t load_two(const char *row, int d, int head_dim) {
  const uint16_t *e = reinterpret_cast<const uint16_t *>(row);
  const uint32_t lo = d < head_dim ? e[d] : 0, hi = d + 1 < head_dim ? e[d + 1] : 0;
  return lo | hi << 16;
}

template <typename T> __device__ __forceinline__ uint32_t pack(float a, float b) {
  typedef T T2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, T2{(T)a, (T)b});
}
template <typename T> __device__ __forceinline__ float unpack(uint32_t x, int half) {
  typedef T T2 __attribute__((ext_vector_type(2)));
  return (float)__builtin_bit_cast(T2, x)[half];
}

// the members of a group: [first, first + n)
struct Members {
  int first, n;
};
__device__ __forceinline__ Members members(const hf_attention &a, int g) {
  const int first = min(max(a.group_offsets[g], 0), a.n_seqs), last = min(max(a.group_offsets[g + 1], first), a.n_seqs);
  return {first, min(last - first, a.max_group)};
}

// How a wavefront finds and reads tiles, and what it does with them.
template <typename T, int kDim, int kMode, bool kLanes, bool kOnce> struct Reader {
  static constexpr int kSteps = kDim / 32; // of the first product
  static constexpr int kOwn = kDim / 16;   // elements of a value row that a lane holds, products of the second kind
  const AttendParams &p;
  const int col = threadIdx.x % 16, grp = threadIdx.x % kWave / 16, in_page = (1 << p.page_shift) - 1;
  // pieces past the head are read from its start, and left out when the result is written
  const uint32_t value_piece = kMode == kPieces && kOwn * col >= p.head_dim ? 0 : 2 * kOwn * col;
  const uint32_t k_lane = kLanes ? 0 : col * (uint32_t)p.token_bytes + 16 * grp;
  const uint32_t v_lane[4] = {first_value(0), first_value(1), first_value(2), first_value(3)};
  const float scale2 = fabsf(p.scale2);

  __device__ __forceinline__ uint32_t first_value(int i) const { return kLanes ? 0 : (4 * grp + i) * (uint32_t)p.token_bytes + value_piece; }

  // the queries of row (counted over the sequences from `first` on) of the rows that read one KV head
  __device__ __forceinline__ void load_queries(u32x4 (&q)[kSteps], int first, int row, int rows, int kv_head) const {
    const int seq = first + row / p.ratio, head = kv_head * p.ratio + row % p.ratio;
    const char *from = static_cast<const char *>(p.a.q) + (seq * p.a.q_stride + head * p.a.q_head_stride) * (int64_t)sizeof(T);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int d = 32 * s + 8 * grp;
      q[s] = u32x4{};
      if constexpr (kMode == kElements) {
        if (row < rows)
          for (int e = 0; e < 4; ++e) q[s][e] = load_two(from, d + 2 * e, p.head_dim);
      } else if (row < rows && (kMode == kWhole || d < p.head_dim)) {
        q[s] = *reinterpret_cast<const u32x4 *>(from + 2 * d);
      }
      if (p.scale2 < 0) q[s] ^= 0x80008000u; // the maximum is taken of the products, so the scale has to be positive
    }
  }

  // Where a tile's tokens are.  A page of 16 tokens or more holds a half of a tile whole, so that its number is the same for all lanes and is
  // fetched and turned into an address by the scalar unit; with smaller pages every lane has its own.
  struct Pages {
    int k[2], v[2];
  };
  struct At {
    int64_t k[2], v[2]; // bytes from the cache's first element
    bool ok[2];
  };
  __device__ __forceinline__ Pages pages_at(const int32_t *table, int token, int end) const {
    Pages g;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (kLanes) {
        g.k[h] = table[min(token + 16 * h + col, end - 1) >> p.page_shift];
        g.v[h] = table[min(token + 16 * h + 4 * grp, end - 1) >> p.page_shift];
      } else {
        g.k[h] = g.v[h] = load_scalar(table + (min(token + 16 * h, end - 1) >> p.page_shift));
      }
    }
    return g;
  }
  // an unusable page number stands for page 0, whose tokens are then not seen
  __device__ __forceinline__ int64_t page_bytes(int page) const { return (int64_t)((uint32_t)page < p.n_pages ? (uint32_t)page : 0u) * p.page_bytes; }
  __device__ __forceinline__ At place(const Pages &g, int token, int kv_head) const {
    const int64_t head = kv_head * p.head_bytes;
    At at;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      at.ok[h] = (uint32_t)g.v[h] < p.n_pages;
      if constexpr (kLanes) {
        at.k[h] = head + page_bytes(g.k[h]) + ((token + 16 * h + col) & in_page) * p.token_bytes + 16 * grp;
        at.v[h] = head + page_bytes(g.v[h]) + ((token + 16 * h + 4 * grp) & in_page) * p.token_bytes + 2 * kOwn * col;
      } else {
        at.k[h] = at.v[h] = head + page_bytes(g.k[h]) + ((token + 16 * h) & in_page) * p.token_bytes;
      }
    }
    return at;
  }

  // what one wavefront alone reads goes past the caches
  static __device__ __forceinline__ u32x4 load16(const char *from) {
    const u32x4 *at = reinterpret_cast<const u32x4 *>(from);
    return kOnce ? __builtin_nontemporal_load(at) : *at;
  }
  __device__ __forceinline__ void load_keys(u32x4 (&k)[2][kSteps], const At &at) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char *row = p.k + at.k[h];
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int d = 32 * s + 8 * grp;
        if constexpr (kMode == kElements) {
          for (int e = 0; e < 4; ++e) k[h][s][e] = load_two(row - 16 * grp, d + 2 * e, p.head_dim);
        } else if constexpr (kMode == kPieces) {
          k[h][s] = u32x4{};
          if (d < p.head_dim) k[h][s] = load16(row + k_lane + 64 * s);
        } else {
          k[h][s] = load16(row + k_lane + 64 * s);
        }
      }
    }
  }
  __device__ __forceinline__ void load_values(uint32_t (&v)[8][kOwn / 2], const At &at) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const char *row = kLanes ? p.v + at.v[h] + i * p.token_bytes : p.v + at.v[h] + v_lane[i];
        if constexpr (kMode == kElements) {
          for (int e = 0; e < kOwn / 2; ++e) v[4 * h + i][e] = load_two(row - 2 * kOwn * col, kOwn * col + 2 * e, p.head_dim);
        } else {
          if constexpr (kLanes) row += (int)value_piece - 2 * kOwn * col;
          if constexpr (kOwn == 4) {
            const u32x2 x = kOnce ? __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(row)) : *reinterpret_cast<const u32x2 *>(row);
            v[4 * h + i][0] = x[0], v[4 * h + i][1] = x[1];
          } else {
#pragma unroll
            for (int e = 0; e < kOwn / 8; ++e) { // the second piece of 16 elements may be past the head too
              const u32x4 x = load16(row + (kMode == kPieces && e && kOwn * col + 8 >= p.head_dim ? 0 : 16 * e));
#pragma unroll
              for (int f = 0; f < 4; ++f) v[4 * h + i][4 * e + f] = x[f];
            }
          }
        }
      }
    }
  }

  // which of the lane's tokens are visible; true if all of the tile's are
  __device__ __forceinline__ bool visible(bool (&seen)[8], const At &at, int token, int end) const {
    const bool whole = token + kTile <= end && (kLanes ? __builtin_amdgcn_ballot_w64(!(at.ok[0] && at.ok[1])) == 0 : at.ok[0] && at.ok[1]);
    if (!whole) {
#pragma unroll
      for (int i = 0; i < 8; ++i) seen[i] = at.ok[i / 4] && token + 16 * (i / 4) + 4 * grp + i % 4 < end;
    }
    return whole;
  }
  static __device__ __forceinline__ void scores(f32x4 (&s)[2], const u32x4 (&k)[2][kSteps], const u32x4 (&q)[kSteps]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      s[h] = f32x4{};
#pragma unroll
      for (int e = 0; e < kSteps; ++e) s[h] = Matrix<T>::product(k[h][e], q[e], s[h]);
    }
  }
  // what is not visible may hold anything, and 0 * NaN is no 0
  static __device__ __forceinline__ void blank(uint32_t (&v)[8][kOwn / 2], const bool (&seen)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < kOwn / 2; ++e) v[i][e] = seen[i] ? v[i][e] : 0;
  }
  // eight tokens of element kOwn * col + j, as a left operand
  static __device__ __forceinline__ u32x4 turned(const uint32_t (&v)[8][kOwn / 2], int j) {
    u32x4 left;
#pragma unroll
    for (int i = 0; i < 4; ++i) left[i] = __builtin_amdgcn_perm(v[2 * i + 1][j / 2], v[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
    return left;
  }
};

// 16 rows' softmax so far; m of the products, before the scale.  m follows the largest score only when one is past it by kSlack of base 2 (P is
// then below 2^kSlack): with 16 rows to a tile some row has a new largest score in nearly every tile, and everything would be rescaled each time.
// In float16 the two halves of P share the type's smallest step, 2^-24, so that weights far below m would lose their bits one by one, where the tokens above
// them may have values of 0 (16 nats below: 6 % off; 18: nothing left).  P carries 2^kUp there, which with the slack stays in the type, and where a row's largest
// score of a tile is kFall below m, m goes down to it: half a step is then 2^-17 of the tile's largest weight at most.  The sums grow by as much, up to
// 2^kSums: a row's weights of less than 2^-45 of their sum show in no float16 output.
template <typename T> constexpr bool kNarrow = std::is_same_v<T, _Float16>;
template <typename T> constexpr float kSlack = kNarrow<T> ? 7 : 8;
template <typename T> constexpr float kUp = kNarrow<T> ? 8 : 0;
constexpr float kFall = 16, kSums = 60;
constexpr float kCoarse = 1 << 22; // scores of base 2 whose own rounding could take P past the type together with the slack
template <typename T, int kOwn> struct Rows {
  f32x4 o[kOwn];
  float m, l, limit; // limit: m and the slack
  __device__ __forceinline__ void clear() {
    m = limit = -INFINITY, l = 0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) o[j] = f32x4{};
  }
  // a tile's scores join the maximum and the sum, and become P in two halves
  __device__ __forceinline__ void join(const f32x4 (&s)[2], bool whole, const bool (&seen)[8], float scale2, u32x4 &hi, u32x4 &lo) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = s[i / 4][i % 4];
    if (!whole) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = seen[i] ? x[i] : -INFINITY;
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
    bool moves = __builtin_amdgcn_ballot_w64(top > limit) != 0;
    if constexpr (kNarrow<T>) { // all four lanes of a column
      uint64_t low = __builtin_amdgcn_ballot_w64(top < limit - (kSlack<T> + kFall) / scale2);
      low &= low >> 32;
      moves |= (low & low >> 16 & 0xFFFF) != 0;
    }
    if (moves) {
      top = over_rows<Max>(top);
      float m_new = fmaxf(m, top);
      if constexpr (kNarrow<T>) {
        const float room = kSums - __builtin_amdgcn_logf(over_rows<Sum>(l));
        if (top < m - kFall / scale2 && top > -INFINITY) m_new = fmaxf(top, m - fmaxf(room, 0.f) / scale2);
      }
      const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m_new) * scale2);
      m = m_new;
      limit = kNarrow<T> && fabsf(m) * scale2 > kCoarse ? m : m + kSlack<T> / scale2;
      l *= keep;
#pragma unroll
      for (int j = 0; j < kOwn; ++j) o[j] *= keep;
    }
    const float base = m == -INFINITY ? 0.f : kNarrow<T> ? kUp<T> - m * scale2 : -m * scale2;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], scale2, base));
    if (!whole) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = seen[i] ? x[i] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) l += x[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      hi[i] = pack<T>(x[2 * i], x[2 * i + 1]);
      lo[i] = pack<T>(x[2 * i] - unpack<T>(hi[i], 0), x[2 * i + 1] - unpack<T>(hi[i], 1));
    }
  }
  __device__ __forceinline__ void add(int j, u32x4 left, u32x4 hi, u32x4 lo) { o[j] = Matrix<T>::product(left, lo, Matrix<T>::product(left, hi, o[j])); }
};

// a row's output and lse from its sums; acc: kN elements from d0 on
template <typename T, int kN, int kMode>
__device__ __forceinline__ void write_row(const AttendParams &p, int seq, int head, int d0, float m2, float sum, const float *acc) {
  const hf_attention &a = p.a;
  const float scale = sum == 0 ? 0.f : 1 / sum;
  T *to = static_cast<T *>(a.out) + seq * a.out_stride + head * a.out_head_stride + d0;
#pragma unroll
  for (int e = 0; e < kN; ++e)
    if (kMode == kWhole || d0 + e < p.head_dim) to[e] = (T)(acc[e] * scale);
  if (a.lse && d0 == 0) a.lse[(int64_t)seq * a.n_q_heads + head] = sum == 0 ? -INFINITY : (m2 + __builtin_amdgcn_logf(sum)) * kLn2;
}
// a row's partial result
template <int kN, int kMode> __device__ __forceinline__ void write_part(const AttendParams &p, int64_t slot, int d0, float top, float m2, float sum, const float *acc) {
  float *to = p.part_o + slot * p.head_dim + d0;
  if constexpr (kMode == kWhole) {
#pragma unroll
    for (int e = 0; e < kN; e += 4) *reinterpret_cast<f32x4 *>(to + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
  } else {
#pragma unroll
    for (int e = 0; e < kN; ++e)
      if (d0 + e < p.head_dim) to[e] = acc[e];
  }
  if (d0 == 0) p.part_ml[2 * slot] = top == -INFINITY ? -INFINITY : m2, p.part_ml[2 * slot + 1] = sum;
}

template <typename T, int kN, int kMode>
__device__ __forceinline__ void write_result(const AttendParams &p, int seq, int head, int part_index, int d0, float top, float scale2, float sum, const float *acc) {
  const float m2 = kNarrow<T> ? top * scale2 - kUp<T> : top * scale2;
  if (p.s.direct) write_row<T, kN, kMode>(p, seq, head, d0, m2, sum, acc);
  else write_part<kN, kMode>(p, ((int64_t)seq * p.a.n_q_heads + head) * (p.s.prefix_parts + p.s.suffix_parts) + part_index, d0, top, m2, sum, acc);
}

// The parts of a workgroup's wavefronts become one: kRowWaves of them have rows of their own, the others the same rows over other tokens.
template <typename T, int kDim, int kWaves, int kQ, int kRowWaves, int kMode>
__device__ __forceinline__ void join_waves(const AttendParams &p, Rows<T, kDim / 16> (&r)[kQ], Members who, int row0, int kv_head, int part_index, float scale2, float *shared) {
  constexpr int kOwn = kDim / 16, kTokenWaves = kWaves / kRowWaves;
  const int rows = who.n * p.ratio, col = threadIdx.x % 16, grp = threadIdx.x % kWave / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), row_wave = wave % kRowWaves, token_wave = wave / kRowWaves;
#pragma unroll
  for (int n = 0; n < kQ; ++n) r[n].l = over_rows<Sum>(r[n].l);
  constexpr int kPitch = kDim + 4, kRows = kRowWaves * kRowsTile;
  float *const both = shared + kTokenWaves * kRows * kPitch; // [token wave, row, 2]
#pragma unroll
  for (int n = 0; n < kQ; ++n) {
    if (n) __syncthreads();
    const int mine = token_wave * kRows + row_wave * kRowsTile + col;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < kOwn; ++j) shared[mine * kPitch + kOwn * (4 * grp + i) + j] = r[n].o[j][i];
    if (grp == 0) both[2 * mine] = r[n].m, both[2 * mine + 1] = r[n].l;
    __syncthreads();
#pragma unroll
    for (int r0 = 0; r0 < kRows; r0 += kWaves * kWave / 16) {
      const int at = r0 + threadIdx.x / 16, d0 = threadIdx.x % 16 * kOwn;
      const int row = row0 + (at / kRowsTile * kQ + n) * kRowsTile + at % kRowsTile;
      if (at < kRows && row < rows) {
        float top = -INFINITY, sum = 0, acc[kOwn] = {};
#pragma unroll
        for (int w = 0; w < kTokenWaves; ++w) top = fmaxf(top, both[2 * (w * kRows + at)]);
#pragma unroll
        for (int w = 0; w < kTokenWaves; ++w) {
          const float mw = both[2 * (w * kRows + at)], weight = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mw - top) * scale2);
          sum += weight * both[2 * (w * kRows + at) + 1];
#pragma unroll
          for (int e = 0; e < kOwn; ++e) acc[e] += weight * shared[(w * kRows + at) * kPitch + d0 + e];
        }
        write_result<T, kOwn, kMode>(p, who.first + row / p.ratio, kv_head * p.ratio + row % p.ratio, part_index, d0, top, scale2, sum, acc);
      }
    }
  }
}

// What the queries q see in the tokens of a segment, a tile at every kStep tokens from `token` on.
template <typename R, typename T, int kDim, int kQ>
__device__ __forceinline__ void sweep(const R &reader, const int32_t *table, int token, int kStep, int end, int kv_head, const u32x4 (&q)[kQ][R::kSteps],
                                      Rows<T, kDim / 16> (&r)[kQ]) {
  // Page numbers are fetched two tiles ahead.  The next tile's keys are on their way from when the scores are made, its values from when they are added
  // up: each is asked for as soon as its registers are free.
  u32x4 k[2][R::kSteps];
  uint32_t v[8][R::kOwn / 2];
  typename R::At at = reader.place(reader.pages_at(table, token, end), token, kv_head);
  typename R::Pages next = reader.pages_at(table, token + kStep, end);
  reader.load_keys(k, at);
  reader.load_values(v, at);
  // (the last tile has code of its own: with a branch around the loads the compiler could not tell how many are on their way, and would wait for all)
  const auto turn = [&](auto more) {
    bool seen[8];
    const bool whole = reader.visible(seen, at, token, end);
    f32x4 s[kQ][2];
#pragma unroll
    for (int n = 0; n < kQ; ++n) R::scores(s[n], k, q[n]);
    if constexpr (more) {
      at = reader.place(next, token + kStep, kv_head);
      next = reader.pages_at(table, token + 2 * kStep, end);
      reader.load_keys(k, at);
    }
    u32x4 hi[kQ], lo[kQ];
#pragma unroll
    for (int n = 0; n < kQ; ++n) r[n].join(s[n], whole, seen, reader.scale2, hi[n], lo[n]);
    if (!whole) R::blank(v, seen);
#pragma unroll
    for (int j = 0; j < R::kOwn; ++j) {
      const u32x4 left = R::turned(v, j);
#pragma unroll
      for (int n = 0; n < kQ; ++n) r[n].add(j, left, hi[n], lo[n]);
    }
    if constexpr (more) reader.load_values(v, at);
  };
  for (; token + kStep < end; token += kStep) turn(std::true_type());
  turn(std::false_type());
}

// Rows row0 .. of a segment (the sequences [first, first + n), all of which see its tokens) over its tokens [begin, end).  kRowWaves wavefronts
// have kQ * 16 rows each, and the others the same rows over other tokens.
template <typename T, int kDim, int kWaves, int kQ, int kRowWaves, int kMode, bool kLanes, bool kOnce>
__device__ __forceinline__ void part(const AttendParams &p, const int32_t *table, int begin, int end, Members who, int row0, int kv_head, int part_index,
                                     float *shared) {
  typedef Reader<T, kDim, kMode, kLanes, kOnce> R;
  constexpr int kTokenWaves = kWaves / kRowWaves;
  const R reader = {p};
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), row_wave = wave % kRowWaves, token_wave = wave / kRowWaves;
  const int rows = who.n * p.ratio, my_row0 = row0 + row_wave * kQ * kRowsTile;

  u32x4 q[kQ][R::kSteps];
  Rows<T, R::kOwn> r[kQ];
#pragma unroll
  for (int n = 0; n < kQ; ++n) {
    reader.load_queries(q[n], who.first, my_row0 + n * kRowsTile + reader.col, rows, kv_head);
    r[n].clear();
  }
  const int token = begin + token_wave * kTile;
  if (token < end && my_row0 < rows) sweep<R, T, kDim, kQ>(reader, table, token, kTokenWaves * kTile, end, kv_head, q, r);
  join_waves<T, kDim, kWaves, kQ, kRowWaves, kMode>(p, r, who, row0, kv_head, part_index, reader.scale2, shared);
}

// The sequence with the n-th longest response (equal ones in order), of at most kThreads.  Workgroups are handed out in order: with the longest first
// the last ones to run are short.
template <int kThreads> __device__ __forceinline__ int nth_longest(const AttendParams &p, int n) {
  __shared__ __attribute__((aligned(16))) int lens[kThreads];
  __shared__ int found;
  const int t = threadIdx.x, own = t < p.a.n_seqs ? max(min(p.a.suffix_lens[t], p.s.max_suffix), 0) : -1;
  lens[t] = own;
  __syncthreads();
  int rank = 0;
  for (int j = 0; j < p.a.n_seqs; j += 4) {
    const int4 x = *reinterpret_cast<const int4 *>(lens + j);
    rank += (x.x > own || (x.x == own && j < t)) + (x.y > own || (x.y == own && j + 1 < t)) + (x.z > own || (x.z == own && j + 2 < t)) +
            (x.w > own || (x.w == own && j + 3 < t));
  }
  if (t < p.a.n_seqs && rank == n) found = t;
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(found);
}

// The parts of prompts and of responses; both in one grid where prompts have few rows too.
template <typename T, int kDim, int kWaves, int kQ, int kRowWaves, int kMode, bool kLanes, bool kOnce>
__global__ __launch_bounds__(kWaves * kWave, kDim > 128 || kMode == kElements ? 1 : kQ > 1 || kDim > 64 ? 2 : 3) void attend_parts(AttendParams p, uint32_t prefix_wgs) {
  __shared__ float shared[kWaves * kRowsTile * (kDim + 4 + 2)];
  const hf_attention &a = p.a;
  uint32_t id = blockIdx.x;
  if (id < prefix_wgs) {
    // the query blocks of a part follow one another on one XCD (workgroups go round over the eight), where L2 holds the part's keys and values for them
    const uint32_t xcd = id % 8, turn = id / 8, block = turn % p.s.prefix_blocks;
    uint32_t item = turn / p.s.prefix_blocks * 8 + xcd;
    const int kv_head = item % p.n_kv_heads;
    item /= p.n_kv_heads;
    const int g = item % a.n_groups, index = item / a.n_groups;
    if (index >= p.s.prefix_parts) return;
    const int begin = index * p.s.prefix_chunk, end = min(min(a.prefix_lens[g], p.s.max_prefix), begin + p.s.prefix_chunk);
    const Members who = members(a, g);
    const int row0 = block * kRowWaves * kQ * kRowsTile;
    if (begin >= end || row0 >= who.n * p.ratio) return;
    part<T, kDim, kWaves, kQ, kRowWaves, kMode, kLanes, kOnce>(p, a.prefix_pages + (int64_t)g * a.prefix_width, begin, end, who, row0, kv_head, index, shared);
  } else {
    id -= prefix_wgs;
    const int kv_head = id % p.n_kv_heads;
    id /= p.n_kv_heads;
    const int block = id % p.s.suffix_blocks;
    id /= p.s.suffix_blocks;
    const int seq = p.s.ordered ? nth_longest<kWaves * kWave>(p, id % a.n_seqs) : id % a.n_seqs, index = id / a.n_seqs;
    const int begin = index * p.s.suffix_chunk, end = min(min(a.suffix_lens[seq], p.s.max_suffix), begin + p.s.suffix_chunk);
    if (begin >= end && !p.s.direct) return;
    part<T, kDim, kWaves, 1, 1, kMode, kLanes, kOnce>(p, a.suffix_pages + (int64_t)seq * a.suffix_width, begin, end, Members{seq, 1}, block * kRowsTile, kv_head,
                                                      p.s.prefix_parts + index, shared);
  }
}

// Responses so short, and so many, that a workgroup for each would do little but start up: a wavefront takes one sequence and KV head, all of its tokens.
template <typename T, int kDim, int kMode, bool kLanes> __global__ __launch_bounds__(kThreads, kDim > 128 || kMode == kElements ? 1 : kDim > 64 ? 2 : 3)
void attend_short(AttendParams p) {
  typedef Reader<T, kDim, kMode, kLanes, true> R;
  constexpr int kSteps = R::kSteps, kOwn = R::kOwn;
  const hf_attention &a = p.a;
  uint32_t id = blockIdx.x * (kThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int kv_head = id % p.n_kv_heads;
  id /= p.n_kv_heads;
  const int row0 = id % p.s.suffix_blocks * kRowsTile, seq = id / p.s.suffix_blocks;
  if (seq >= a.n_seqs) return;
  const int end = min(load_scalar(a.suffix_lens + seq), p.s.max_suffix);
  if (end <= 0 && !p.s.direct) return;
  const R reader = {p};
  const int32_t *table = a.suffix_pages + (int64_t)seq * a.suffix_width;
  u32x4 q[kSteps];
  Rows<T, kOwn> r;
  reader.load_queries(q, seq, row0 + reader.col, p.ratio, kv_head);
  r.clear();
  for (int token = 0; token < end; token += kTile) {
    u32x4 k[2][kSteps];
    uint32_t v[8][kOwn / 2];
    const typename R::At at = reader.place(reader.pages_at(table, token, end), token, kv_head);
    reader.load_keys(k, at);
    reader.load_values(v, at);
    bool seen[8];
    const bool whole = reader.visible(seen, at, token, end);
    f32x4 s[2];
    R::scores(s, k, q);
    u32x4 hi, lo;
    r.join(s, whole, seen, reader.scale2, hi, lo);
    if (!whole) R::blank(v, seen);
#pragma unroll
    for (int j = 0; j < kOwn; ++j) r.add(j, R::turned(v, j), hi, lo);
  }
  const float sum = over_rows<Sum>(r.l);
  const int row = row0 + reader.col;
  if (row >= p.ratio) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float acc[kOwn];
#pragma unroll
    for (int j = 0; j < kOwn; ++j) acc[j] = r.o[j][i];
    write_result<T, kOwn, kMode>(p, seq, kv_head * p.ratio + row, p.s.prefix_parts, kOwn * (4 * reader.grp + i), r.m, reader.scale2, sum, acc);
  }
}

// Few and short contexts, in one launch: a workgroup takes a sequence and KV head, its wavefronts the tiles of prompt and response in turn.
// (Eight wavefronts were level or slower: 13.4 against 15.8 us with 512 workgroups of 512 tokens.)
template <typename T, int kDim, int kMode, bool kLanes>
__global__ __launch_bounds__(kThreads, kDim > 128 || kMode == kElements ? 1 : 2) void attend_small(AttendParams p) {
  constexpr int kWaves = kThreads / kWave;
  typedef Reader<T, kDim, kMode, kLanes, false> R;
  __shared__ float shared[kWaves * kRowsTile * (kDim + 4 + 2)];
  const hf_attention &a = p.a;
  uint32_t id = blockIdx.x;
  const int kv_head = id % p.n_kv_heads;
  id /= p.n_kv_heads;
  const int row0 = id % p.s.suffix_blocks * kRowsTile, seq = id / p.s.suffix_blocks;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const R reader = {p};
  u32x4 q[1][R::kSteps];
  Rows<T, R::kOwn> r[1];
  reader.load_queries(q[0], seq, row0 + reader.col, p.ratio, kv_head);
  r[0].clear();
  const int own = min(load_scalar(a.suffix_lens + seq), p.s.max_suffix);
  int prompt = -1;
  for (int g0 = 0; g0 < a.n_groups && prompt < 0; g0 += kWave) { // every lane asks for another prompt whether the sequence is one of its samples
    const int g = g0 + (int)(threadIdx.x % kWave);
    const Members who = members(a, min(g, a.n_groups - 1));
    const uint64_t its = __builtin_amdgcn_ballot_w64(g < a.n_groups && seq >= who.first && seq < who.first + who.n);
    if (its) prompt = g0 + __builtin_ctzll(its);
  }
  int tiles = 0;
  if (prompt >= 0) {
    const int end = min(load_scalar(a.prefix_lens + prompt), p.s.max_prefix);
    tiles = max(end + kTile - 1, 0) / kTile;
    if (wave * kTile < end)
      sweep<R, T, kDim, 1>(reader, a.prefix_pages + (int64_t)prompt * a.prefix_width, wave * kTile, kWaves * kTile, end, kv_head, q, r);
  }
  const int token = (wave + kWaves - tiles % kWaves) % kWaves * kTile; // on with the wavefront whose turn it is
  if (token < own) sweep<R, T, kDim, 1>(reader, a.suffix_pages + (int64_t)seq * a.suffix_width, token, kWaves * kTile, own, kv_head, q, r);
  join_waves<T, kDim, kWaves, 1, 1, kMode>(p, r, Members{seq, 1}, row0, kv_head, 0, reader.scale2, shared);
}

// A row (sequence, query head) out of its parts, in order.  kDim / 4 lanes have four elements of it each; `split` such teams share a row's parts
// where these are many, each taking every split-th.  Bound by latency: 3.4 us for 16 rows of two parts, 7.7 for 976 rows of 36, 8.5 for 8192 rows of five.
template <typename T, int kDim> __global__ __launch_bounds__(kThreads) void attend_merge(AttendParams p, int split) {
  constexpr int kTeam = kDim / 4, kTeams = kThreads / kTeam;
  __shared__ f32x4 shared[kThreads];
  const hf_attention &a = p.a;
  const int lane = threadIdx.x % kTeam, team = threadIdx.x / kTeam, share = team % split;
  const int n_rows = a.n_seqs * a.n_q_heads, at = blockIdx.x * (kTeams / split) + team / split, row = min(at, n_rows - 1);
  const int seq = row / a.n_q_heads, head = row % a.n_q_heads;
  int n_prefix = 0;
  if (p.s.prefix_parts) {
    int len = 0;
    for (int g0 = 0; g0 < a.n_groups; g0 += kTeam) { // every lane asks for another prompt whether the sequence is one of its samples
      const int g = min(g0 + lane, a.n_groups - 1);
      const Members who = members(a, g);
      const int its = a.prefix_lens[g];
      if (seq >= who.first && seq < who.first + who.n) len = its;
    }
#pragma unroll
    for (int d = 1; d < kTeam; d *= 2) len = max(len, __shfl_xor(len, d)); // the others have 0
    n_prefix = (min(len, p.s.max_prefix) + p.s.prefix_chunk - 1) / p.s.prefix_chunk;
  }
  const int own = min(a.suffix_lens[seq], p.s.max_suffix), n_suffix = own > 0 ? (own + p.s.suffix_chunk - 1) / p.s.suffix_chunk : 0;
  const int n = n_prefix + n_suffix;
  const int64_t slot0 = (int64_t)row * (p.s.prefix_parts + p.s.suffix_parts);
  const auto slot = [&](int i) { return slot0 + (i < n_prefix ? i : p.s.prefix_parts + i - n_prefix); };
  float top = -INFINITY;
  for (int i = lane; i < n; i += kTeam) top = fmaxf(top, p.part_ml[2 * slot(i)]);
#pragma unroll
  for (int d = 1; d < kTeam; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  const int d0 = 4 * lane;
  const bool aligned = p.head_dim % 4 == 0;
  const auto load = [&](int i) {
    const float *from = p.part_o + slot(i) * p.head_dim + d0;
    f32x4 x = {};
    if (aligned) {
      if (d0 < p.head_dim) x = *reinterpret_cast<const f32x4 *>(from);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (d0 + e < p.head_dim) x[e] = from[e];
    }
    return x;
  };
  f32x4 acc = {};
  float sum = 0;
  for (int i0 = 0; i0 < n; i0 += kTeam) {
    const int i = i0 + lane;
    float weight = 0;
    if (i < n) {
      const float m = p.part_ml[2 * slot(i)];
      weight = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
      sum += weight * p.part_ml[2 * slot(i) + 1];
    }
    const int last = min(kTeam, n - i0);
    for (int j = share; j < last; j += split) acc += __shfl(weight, j, kTeam) * load(i0 + j);
  }
#pragma unroll
  for (int d = 1; d < kTeam; d *= 2) sum += __shfl_xor(sum, d);
  if (split > 1) {
    shared[threadIdx.x] = acc;
    __syncthreads();
    if (share) return;
    for (int k = 1; k < split; ++k) acc += shared[threadIdx.x + k * kTeam];
  }
  if (at >= n_rows) return;
  const float scale = sum == 0 ? 0.f : 1 / sum;
  T *to = static_cast<T *>(a.out) + seq * a.out_stride + head * a.out_head_stride + d0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (d0 + e < p.head_dim) to[e] = (T)(acc[e] * scale);
  if (a.lse && lane == 0) a.lse[row] = sum == 0 ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <typename T, int kDim, int kMode, bool kLanes> hipError_t launch_mode(const AttendParams &p, const AttendLaunch &s, hipStream_t st) {
  if (s.small) return enqueue_kernel(attend_small<T, kDim, kMode, kLanes>, dim3((uint32_t)s.suffix_wgs), kThreads, st, p);
  uint32_t prefix_wgs = (uint32_t)s.prefix_wgs, suffix_wgs = (uint32_t)s.suffix_wgs;
  hipError_t e = hipSuccess;
  if constexpr (kDim <= 128 && kMode != kElements) {
    if (s.row_waves) {
      const auto prompts = [&](auto kernel) { return enqueue_kernel(kernel, dim3(prefix_wgs + (s.together ? suffix_wgs : 0)), 8 * kWave, st, p, prefix_wgs); };
      e = s.row_waves == 4   ? prompts(attend_parts<T, kDim, 8, 2, 4, kMode, kLanes, false>)
          : s.row_waves == 2 ? prompts(attend_parts<T, kDim, 8, 2, 2, kMode, kLanes, false>)
                             : prompts(attend_parts<T, kDim, 8, 2, 1, kMode, kLanes, false>);
      prefix_wgs = 0;
      if (s.together) suffix_wgs = 0;
    }
  }
  if (s.brief) {
    if (e == hipSuccess && prefix_wgs) e = enqueue_kernel(attend_parts<T, kDim, 4, 1, 1, kMode, kLanes, true>, dim3(prefix_wgs), 4 * kWave, st, p, prefix_wgs);
    if (e == hipSuccess) e = enqueue_kernel(attend_short<T, kDim, kMode, kLanes>, dim3((suffix_wgs + 3) / 4), kThreads, st, p);
  } else if (e == hipSuccess && prefix_wgs + suffix_wgs) {
    e = enqueue_kernel(attend_parts<T, kDim, 4, 1, 1, kMode, kLanes, true>, dim3(prefix_wgs + suffix_wgs), 4 * kWave, st, p, prefix_wgs);
  }
  if (e != hipSuccess || s.direct) return e;
  return enqueue_kernel(attend_merge<T, kDim>, dim3((uint32_t)s.merge_wgs), kThreads, st, p, s.merge_split);
}
template <typename T, int kDim> hipError_t launch_dim(const AttendParams &p, const AttendLaunch &s, bool vec, hipStream_t st) {
  if (!vec) return launch_mode<T, kDim, kElements, true>(p, s, st);
  if (p.head_dim != kDim) return launch_mode<T, kDim, kPieces, true>(p, s, st);
  return s.lanes ? launch_mode<T, kDim, kWhole, true>(p, s, st) : launch_mode<T, kDim, kWhole, false>(p, s, st);
}
template <typename T> hipError_t launch_type(const AttendParams &p, const AttendLaunch &s, bool vec, hipStream_t st) {
  if (p.head_dim <= 64) return launch_dim<T, 64>(p, s, vec, st);
  if (p.head_dim <= 128) return launch_dim<T, 128>(p, s, vec, st);
  return launch_dim<T, 256>(p, s, vec, st);
}

} // namespace

constexpr uint64_t kResident = 3 * 256; // workgroups of four wavefronts that the chip holds

AttendLaunch attend_shape(const hf_kv_cache &cache, const hf_attention &a, bool vec) {
  AttendLaunch s = {};
  const int64_t page = cache.page_tokens, ratio = a.n_q_heads / cache.n_kv_heads;
  s.max_suffix = (int32_t)std::min<int64_t>(a.max_suffix, std::min<int64_t>(a.suffix_width * page, 1 << 30));
  s.max_prefix = a.n_groups ? (int32_t)std::min<int64_t>(a.max_prefix, std::min<int64_t>(a.prefix_width * page, 1 << 30)) : 0;
  // Parts are as long as they may be while there are 1024 workgroups.  A workgroup starts up for some 5 us (length, page numbers, first tiles one after another) and
  // every part costs its rows a partial result.  us at 1 / 2 / 4 / 8 parts a response, 128 responses of 2048 tokens (8 KV heads, eight rows each) 165 / 178 /
  // 198 / 237, of 1 to 2048 tokens 94 / 104 / 114 / 140.
  const auto chunk = [&](int64_t len, int64_t others) {
    int64_t c = 128;
    while (c < len && others * ((len + 2 * c - 1) / (2 * c)) >= 1024) c *= 2;
    return (int32_t)c;
  };
  // Prompts with many rows: a CU holds one workgroup, which takes 12 us and 30 ns a token of 128 rows (half of that for every half of the rows), and a part costs a row 0.26 ns
  // in writing and merging.  us at 1 / 2 / 4 / 8 / 16 / 32 / 64 parts a prompt, responses of one token, and in brackets what the sum of these costs takes:
  //   1 prompt x 2 KV heads, 488 rows of 32749 tokens  1109 / 564 / 294 / 155 / 87 / 58 / 66 (56)     1 x 8, 64 rows of 8192  147 / 81 / 47 / 30 / 22.0 / 23.1 / 31 (22.8)
  //   8 x 8, 128 rows of 2048  91 / 59 / 45 / 55 / 79 (44)                                            2 x 32, 20 rows of 4096  56 / 41 / 39 / 45 / 57 / 73 (39)
  //   16 x 2, 96 rows of 1024  42 / 31 / 27.3 / 28.3 (28.0)                                           32 x 8, 512 rows of 512  206 / 251 / 352 (206)
  //   1 x 12, 40 rows of 32768, heads of 64  340 / 180 / 99 / 58 / 38 / 42 / 43 (34)                  1 x 8, 40 rows of 20000, heads of 72  265 / 141 / 79 / 46 / 30 / 27 / 32 (26)
  // It is within 4 % of the best power of two there and on four more shapes.
  const auto chunk_of_prompts = [&](int64_t len, int64_t others, int row_waves) {
    int64_t best = 0;
    double least = 0;
    for (int64_t n = 1; n <= 256; n += n < 16 ? 1 : n / 8) {
      const int64_t c = std::max<int64_t>((len + n * 128 - 1) / (n * 128) * 128, 128), parts = (len + c - 1) / c;
      const double us = (double)((others * parts + 255) / 256) * (12 + 0.0075 * row_waves * (double)c) + 2.6e-4 * (double)parts * a.n_seqs * a.n_q_heads;
      if (best == 0 || us < least) best = c, least = us;
      if (c == 128) break;
    }
    return (int32_t)best;
  };
  const int64_t rows = std::min<int64_t>(a.max_group, a.n_seqs) * ratio;
  const bool two = vec && cache.head_dim <= 128 && rows > kRowsTile;
  s.row_waves = !two ? 0 : rows <= 2 * kRowsTile ? 1 : rows <= 4 * kRowsTile ? 2 : 4;
  s.lanes = page < 16 || cache.token_stride >= 1 << 25;
  const int64_t rows_of_wg = two ? 2 * s.row_waves * kRowsTile : kRowsTile;
  s.prefix_blocks = (int32_t)((rows + rows_of_wg - 1) / rows_of_wg);
  s.suffix_blocks = (int32_t)((ratio + kRowsTile - 1) / kRowsTile);
  s.suffix_chunk = chunk(s.max_suffix, (int64_t)a.n_seqs * cache.n_kv_heads * s.suffix_blocks);
  const int64_t prompts = (int64_t)a.n_groups * cache.n_kv_heads * s.prefix_blocks;
  s.prefix_chunk = two ? chunk_of_prompts(s.max_prefix, prompts, s.row_waves) : chunk(s.max_prefix, prompts);
  s.suffix_parts = std::max(1, (s.max_suffix + s.suffix_chunk - 1) / s.suffix_chunk);
  s.prefix_parts = rows ? (s.max_prefix + s.prefix_chunk - 1) / s.prefix_chunk : 0;
  if (s.prefix_parts == 0) s.row_waves = 0;
  s.direct = s.prefix_parts == 0 && s.suffix_parts == 1;
  const uint64_t items = (uint64_t)a.n_groups * s.prefix_parts * cache.n_kv_heads;
  s.prefix_wgs = (items + 7) / 8 * 8 * s.prefix_blocks;
  s.suffix_wgs = (uint64_t)a.n_seqs * s.suffix_parts * s.suffix_blocks * cache.n_kv_heads;
  // where more workgroups than the chip holds at a time have lengths of their own (above: 94 us, 107 in the order of the sequences; 165 against 164 where all are alike)
  s.ordered = a.n_seqs <= kThreads && s.suffix_wgs > kResident && s.max_suffix > 4 * kTile * 4;
  // A wavefront to a short response.  us, four wavefronts / one, lengths from 1 to the bound: heads of 64 and 32 up to 128 tokens 40 / 38 (6144 workgroups) and 28 / 24 (4096), up to
  // 256 53 / 59 and 32.6 / 33.5; heads of 128 up to 32 tokens 20.9 / 18.8 (1536), up to 128 26.8 / 28.1 (1024) and 48.4 / 49.4 (4096), up to 256 33 / 37 and 66 / 75; fewer workgroups than
  // the chip holds, up to 128 tokens, 22 / 27 (768) and, up to 64, 11.5 / 18 (128).  At heads of 128 the limit could be half of this.
  s.brief = s.suffix_wgs > kResident && s.max_suffix <= 4 * kTile;
  // Responses behind the prompts in one grid, in workgroups as large as the prompts'.  us, a grid each / one, by the workgroups of responses: 64 22.6 / 18.0, 488 62.4 / 61.6, 576 37 / 30,
  // 960 18.1 / 17.6; 1024 of up to 512 tokens 36 / 29, 49 / 49 and 52 / 50, of up to 2048 65 / 70, 101 / 116 and 131 / 155; 1280 57 / 53, 1920 22.6 / 23.5.  Up to 256 it was never slower.
  s.together = s.row_waves && !s.brief && s.suffix_wgs <= 256;
  if (!s.direct) s.workspace = ((size_t)a.n_seqs * a.n_q_heads * (s.prefix_parts + s.suffix_parts)) * (cache.head_dim + 2) * sizeof(float);
  // (the workspace stays as it is asked for by the parts, so that it follows from those alone)
  // One launch over whole contexts saves the merge and its launch, and reads a prompt once for every sample, from L2; a workgroup takes 3 us and 9 ns a token of 128
  // elements.  us, parts / one launch: 16 workgroups (sequence, KV head) of 164 tokens 8.5 / 5.6, 64 of 512 9.7 / 7.9, of 1024 11.5 / 11.9, 32 of 768 9.5 / 10.3, 256 of 1024
  // 22 / 14, 512 of 1024 23 / 21, 1024 of 512 27 / 23, of 1024 28 / 40, 2048 of 256 35 / 28, of 512 40 / 44; single elements, 64 of 128 17 / 13, of 256 17 / 21.
  const int64_t tokens = (int64_t)s.max_prefix + s.max_suffix, one = (int64_t)a.n_seqs * s.suffix_blocks * cache.n_kv_heads;
  const int64_t padded = cache.head_dim <= 64 ? 64 : cache.head_dim <= 128 ? 128 : 256;
  s.small = !s.direct && tokens <= (vec ? (one < 128 ? 640 : 1024) * 128 / padded : 128) && one * tokens <= 1 << 19;
  if (s.small) s.direct = true, s.prefix_wgs = 0, s.suffix_wgs = one, s.row_waves = 0, s.brief = s.together = false;
  s.merge_split = 1;
  const int64_t teams = kThreads / (padded / 4);
  while (s.merge_split < teams && 4 * s.merge_split < s.prefix_parts + s.suffix_parts) s.merge_split *= 2;
  const int64_t rows_of_merge = teams / s.merge_split;
  s.merge_wgs = s.direct ? 0 : ((int64_t)a.n_seqs * a.n_q_heads + rows_of_merge - 1) / rows_of_merge;
  // what launch_mode starts
  const uint64_t shared = s.row_waves ? s.prefix_wgs + (s.together ? s.suffix_wgs : 0) : 0;
  const uint64_t parts = s.together ? 0 : (s.row_waves ? 0 : s.prefix_wgs) + (s.brief ? 0 : s.suffix_wgs), brief = s.brief ? (s.suffix_wgs + 3) / 4 : 0;
  s.fits = shared <= kMaxWgs / 2 && parts <= kMaxWgs && brief <= kMaxWgs && s.merge_wgs <= kMaxWgs;
  return s;
}

int launch_attend(const hf_kv_cache &cache, const hf_attention &a, const AttendLaunch &s, bool vec, void *stream) {
  AttendParams p = {a, s, static_cast<const char *>(cache.k), static_cast<const char *>(cache.v), 2 * cache.page_stride, 2 * cache.head_stride,
                    2 * cache.token_stride, (uint32_t)cache.n_pages,
                    cache.n_kv_heads, cache.head_dim, __builtin_ctz(cache.page_tokens), a.n_q_heads / cache.n_kv_heads, a.scale * kLog2e, nullptr, nullptr};
  if (!s.direct) {
    p.part_o = static_cast<float *>(a.workspace);
    p.part_ml = p.part_o + (size_t)a.n_seqs * a.n_q_heads * (s.prefix_parts + s.suffix_parts) * cache.head_dim;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  return (int)(cache.dtype == HF_BF16 ? launch_type<__bf16>(p, s, vec, st) : launch_type<_Float16>(p, s, vec, st));
}

} // namespace hf
