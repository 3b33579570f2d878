// Attention of one query token per sequence over a paged cache, the samples of a prompt taking the prompt's pages together.
//
//   x_j = scale <q, k_j>,  m = max_j x_j,  l = sum_j exp(x_j - m),  o = sum_j exp(x_j - m) v_j / l
//
// Any cut of the tokens into parts gives (m, l, o) of each part, and parts merge exactly:
// m = max m_i, l = sum l_i exp(m_i - m), o likewise.  A prompt is cut into parts whose rows are all the queries of its samples that
// read one KV head (samples x query heads per KV head), a response into parts whose rows are the sequence's own query heads, and a
// second kernel merges a row's parts in a fixed order.
//
// Bound: a response's keys and values are read for one sequence alone, 4 bytes per (token, element) for 4 x rows operations, so
// HBM is the bound there; a prompt's for all of its samples' rows.  What keeps the loads wide and the wavefronts fed:
//  - a wavefront takes tiles of 32 tokens straight from memory into registers, the next tile's loads in flight while
//    it works on the present one; nothing is staged and no wavefront waits for another until its part is done;
//  - scores are made transposed, S^T = K Q^T: the accumulator then holds, for the query of a lane's column, four tokens of each 16, which
//    is what the second product O^T = V^T P^T wants as its right operand if its 32 tokens are taken in the order (16-token
//    half, lane group, token): P never moves between lanes;
//  - a lane loads 16 bytes of each of its eight tokens' values, whole rows over 16 lanes; the eight rows are turned in its registers (one byte
//    permute per two elements) into left operands for eight products, product j holding every eighth element of a head.
// Exponentials are of base 2, the scale carries the factor.  P is rounded to the cache's type twice, once for its upper bits and once for the
// rest: rounded once it would add as much to the error as the rounding of the output does.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "rollout_kernels.hpp"

namespace hf {

namespace {

constexpr int kThreads = 256, kWave = 64, kWaves = kThreads / kWave;
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
  const void *k, *v;
  int64_t page_stride, head_stride, token_stride;
  uint32_t n_pages;
  int32_t n_kv_heads, head_dim, page_shift, ratio;
  float scale2;   // of base 2
  float *part_o;  // [row, part, head_dim]
  float *part_ml; // [row, part, 2]
};

// How heads are read: whole (head_dim is the kernel's), in pieces of 8 elements, or by single elements
enum { kWhole = 0, kPieces = 1, kElements = 2 };

// kN elements (a multiple of 4, at most 8) from d on; zeros past the head
template <typename T, int kN, int kMode> __device__ __forceinline__ void load(uint32_t *to, const T *row, int d, int head_dim) {
  if constexpr (kMode == kElements) {
#pragma unroll
    for (int e = 0; e < kN; e += 2) {
      const uint32_t lo = d + e < head_dim ? __builtin_bit_cast(uint16_t, row[d + e]) : 0, hi = d + e + 1 < head_dim ? __builtin_bit_cast(uint16_t, row[d + e + 1]) : 0;
      to[e / 2] = lo | hi << 16;
    }
  } else {
    const bool in = kMode == kWhole || d < head_dim;
    if constexpr (kN == 8) {
      const u32x4 x = in ? *reinterpret_cast<const u32x4 *>(row + d) : u32x4{};
#pragma unroll
      for (int e = 0; e < 4; ++e) to[e] = x[e];
    } else {
      const u32x2 x = in ? *reinterpret_cast<const u32x2 *>(row + d) : u32x2{};
#pragma unroll
      for (int e = 0; e < 2; ++e) to[e] = x[e];
    }
  }
}

// x of a lane and of the lane 32 (16) further, in either order: the instruction exchanges the upper half (odd rows of 16) of one register with the
// lower half (even rows) of the other.  Written by hand because the compiler's builtin gives its first result for both; the two
// wait states are those it puts between a write of the operands and the exchange.
__device__ __forceinline__ void swap32(float &a, float &b) { asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b)); }
__device__ __forceinline__ void swap16(float &a, float &b) { asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b)); }
// the largest of the four lanes that share a column, and their sum
__device__ __forceinline__ float column_max(float x) {
  float y = x;
  swap32(x, y);
  x = y = fmaxf(x, y);
  swap16(x, y);
  return fmaxf(x, y);
}
__device__ __forceinline__ float column_sum(float x) {
  float y = x;
  swap32(x, y);
  x = y = x + y;
  swap16(x, y);
  return x + y;
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

// Rows row0 .. of a segment (the sequences [first, first + n), all of which see its tokens) over its tokens [begin, end).
template <typename T, int kDim, int kQ, int kMode>
__device__ __forceinline__ void part(const AttendParams &p, const int32_t *table, int begin, int end, Members who, int row0, int kv_head, int part_index,
                                     float *shared) {
  constexpr int kSteps = kDim / 32; // of the first product
  constexpr int kOwn = kDim / 16;   // elements of a value row that a lane holds, products of the second kind
  constexpr int kPiece = kOwn < 8 ? kOwn : 8;
  const hf_attention &a = p.a;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, col = lane % 16, grp = lane / 16;
  const int rows = who.n * p.ratio;
  const T *keys = static_cast<const T *>(p.k) + kv_head * p.head_stride, *values = static_cast<const T *>(p.v) + kv_head * p.head_stride;
  const int in_page = (1 << p.page_shift) - 1;

  u32x4 q[kQ][kSteps];
#pragma unroll
  for (int n = 0; n < kQ; ++n) {
    const int row = row0 + n * kRowsTile + col;
    const int seq = who.first + row / p.ratio, head = kv_head * p.ratio + row % p.ratio;
    const T *from = static_cast<const T *>(a.q) + seq * a.q_stride + head * a.q_head_stride;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      uint32_t x[4] = {};
      if (row < rows) load<T, 8, kMode>(x, from, 32 * s + 8 * grp, p.head_dim);
      q[n][s] = u32x4{x[0], x[1], x[2], x[3]};
    }
  }

  struct Pages {
    int k[2], v[2]; // of token col and of tokens 4 * grp .. + 3, of either half of a tile; -1 = not visible
  };
  struct Tile {
    uint32_t k[2][kSteps][4], v[8][kOwn / 2];
    int seen[2]; // how many of the lane's four tokens are visible
  };
  const auto page_of = [&](int token) {
    if (token >= end) return -1;
    const int page = table[token >> p.page_shift];
    return (uint32_t)page < p.n_pages ? page : -1;
  };
  const auto pages_at = [&](int token) {
    Pages g;
#pragma unroll
    for (int h = 0; h < 2; ++h) g.k[h] = page_of(token + 16 * h + col), g.v[h] = page_of(token + 16 * h + 4 * grp);
    return g;
  };
  // places that are not visible are read from page 0 and not used
  const auto load_tile = [&](Tile &t, const Pages &g, int token) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const T *row = keys + max(g.k[h], 0) * p.page_stride + ((token + 16 * h + col) & in_page) * p.token_stride;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) load<T, 8, kMode>(t.k[h][s], row, 32 * s + 8 * grp, p.head_dim);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int first = token + 16 * h + 4 * grp;
      t.seen[h] = g.v[h] < 0 ? 0 : min(end - first, 4);
      const T *row = values + max(g.v[h], 0) * p.page_stride + (first & in_page) * p.token_stride;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int e = 0; e < kOwn; e += kPiece) load<T, kPiece, kMode>(t.v[4 * h + i] + e / 2, row + i * p.token_stride, kOwn * col + e, p.head_dim);
      }
    }
  };

  f32x4 o[kQ][kOwn];
  float m[kQ], l[kQ];
#pragma unroll
  for (int n = 0; n < kQ; ++n) {
    m[n] = -INFINITY, l[n] = 0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) o[n][j] = f32x4{};
  }

  const auto use_tile = [&](Tile &t) {
    const bool whole = __builtin_amdgcn_ballot_w64(t.seen[0] < 4 || t.seen[1] < 4) == 0;
    if (!whole) { // what is not visible may hold anything, and 0 * NaN is no 0
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i % 4 >= t.seen[i / 4]) {
#pragma unroll
          for (int e = 0; e < kOwn / 2; ++e) t.v[i][e] = 0;
        }
    }
    u32x4 hi[kQ], lo[kQ];
#pragma unroll
    for (int n = 0; n < kQ; ++n) {
      f32x4 s[2] = {};
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < kSteps; ++e) s[h] = Matrix<T>::product(u32x4{t.k[h][e][0], t.k[h][e][1], t.k[h][e][2], t.k[h][e][3]}, q[n][e], s[h]);
      float x[8], top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = s[i / 4][i % 4] * p.scale2;
        if (!whole && i % 4 >= t.seen[i / 4]) x[i] = -INFINITY;
        top = fmaxf(top, x[i]);
      }
      const float m_new = fmaxf(m[n], column_max(top));
      if (__builtin_amdgcn_ballot_w64(m_new > m[n]) != 0) {
        const float down = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[n] - m_new);
        m[n] = m_new;
        l[n] *= down;
#pragma unroll
        for (int j = 0; j < kOwn; ++j) o[n][j] *= down;
      }
      const float at = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = __builtin_amdgcn_exp2f(x[i] - at);
        l[n] += x[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        hi[n][i] = pack<T>(x[2 * i], x[2 * i + 1]);
        lo[n][i] = pack<T>(x[2 * i] - unpack<T>(hi[n][i], 0), x[2 * i + 1] - unpack<T>(hi[n][i], 1));
      }
    }
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      u32x4 left;
#pragma unroll
      for (int i = 0; i < 4; ++i) left[i] = __builtin_amdgcn_perm(t.v[2 * i + 1][j / 2], t.v[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int n = 0; n < kQ; ++n) o[n][j] = Matrix<T>::product(left, lo[n], Matrix<T>::product(left, hi[n], o[n][j]));
    }
  };

  // page numbers are fetched two tiles ahead, keys and values one, where the registers hold a second tile
  constexpr bool kAhead = kDim <= 128 && kMode != kElements;
  constexpr int kStep = kWaves * kTile;
  int token = begin + wave * kTile;
  if constexpr (kAhead) {
    if (token < end) {
      Tile even, odd;
      Pages next = pages_at(token);
      load_tile(even, next, token);
      next = pages_at(token + kStep);
      for (;;) {
        if (token + kStep < end) {
          load_tile(odd, next, token + kStep);
          next = pages_at(token + 2 * kStep);
        }
        use_tile(even);
        token += kStep;
        if (token >= end) break;
        if (token + kStep < end) {
          load_tile(even, next, token + kStep);
          next = pages_at(token + 2 * kStep);
        }
        use_tile(odd);
        token += kStep;
        if (token >= end) break;
      }
    }
  } else {
    for (; token < end; token += kStep) {
      Tile t;
      load_tile(t, pages_at(token), token);
      use_tile(t);
    }
  }

  // the four wavefronts' parts become one
  constexpr int kPitch = kDim + 4;
  float *const both = shared + kWaves * kRowsTile * kPitch; // [wave, row, 2]
#pragma unroll
  for (int n = 0; n < kQ; ++n) {
    if (n) __syncthreads();
    l[n] = column_sum(l[n]);
    float *mine = shared + (wave * kRowsTile + col) * kPitch;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < kOwn; ++j) mine[kOwn * (4 * grp + i) + j] = o[n][j][i];
    if (grp == 0) both[(wave * kRowsTile + col) * 2] = m[n], both[(wave * kRowsTile + col) * 2 + 1] = l[n];
    __syncthreads();
    const int r = threadIdx.x / 16, d0 = threadIdx.x % 16 * kOwn, row = row0 + n * kRowsTile + r;
    if (row < rows) {
      float top = -INFINITY, sum = 0, acc[kOwn] = {};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, both[(w * kRowsTile + r) * 2]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float mw = both[(w * kRowsTile + r) * 2], weight = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - top);
        sum += weight * both[(w * kRowsTile + r) * 2 + 1];
#pragma unroll
        for (int e = 0; e < kOwn; ++e) acc[e] += weight * shared[(w * kRowsTile + r) * kPitch + d0 + e];
      }
      const int seq = who.first + row / p.ratio, head = kv_head * p.ratio + row % p.ratio;
      const int64_t at = (int64_t)seq * a.n_q_heads + head;
      if (p.s.direct) {
        const float scale = sum == 0 ? 0.f : 1 / sum;
        T *to = static_cast<T *>(a.out) + seq * a.out_stride + head * a.out_head_stride;
#pragma unroll
        for (int e = 0; e < kOwn; ++e)
          if (d0 + e < p.head_dim) to[d0 + e] = (T)(acc[e] * scale);
        if (a.lse && d0 == 0) a.lse[at] = sum == 0 ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
      } else {
        const int64_t slot = at * (p.s.prefix_parts + p.s.suffix_parts) + part_index;
#pragma unroll
        for (int e = 0; e < kOwn; ++e)
          if (d0 + e < p.head_dim) p.part_o[slot * p.head_dim + d0 + e] = acc[e];
        if (d0 == 0) p.part_ml[2 * slot] = top, p.part_ml[2 * slot + 1] = sum;
      }
    }
  }
}

template <typename T, int kDim, int kQ, int kMode> __global__ __launch_bounds__(kThreads, kDim > 128 ? 1 : 2) void attend_parts(AttendParams p) {
  __shared__ float shared[kWaves * kRowsTile * (kDim + 4 + 2)];
  const hf_attention &a = p.a;
  uint32_t id = blockIdx.x;
  if (id < p.s.prefix_wgs) {
    // the query blocks of a part follow one another on one XCD (workgroups go round over the eight), where L2 holds the part's keys and values for them
    const uint32_t xcd = id % 8, turn = id / 8, block = turn % p.s.prefix_blocks;
    uint32_t item = turn / p.s.prefix_blocks * 8 + xcd;
    const int kv_head = item % p.n_kv_heads;
    item /= p.n_kv_heads;
    const int index = item % p.s.prefix_parts, g = item / p.s.prefix_parts;
    if (g >= a.n_groups) return;
    const int begin = index * p.s.prefix_chunk, end = min(min(a.prefix_lens[g], p.s.max_prefix), begin + p.s.prefix_chunk);
    const Members who = members(a, g);
    const int row0 = block * kQ * kRowsTile;
    if (begin >= end || row0 >= who.n * p.ratio) return;
    part<T, kDim, kQ, kMode>(p, a.prefix_pages + (int64_t)g * a.prefix_width, begin, end, who, row0, kv_head, index, shared);
  } else {
    id -= p.s.prefix_wgs;
    const int kv_head = id % p.n_kv_heads;
    id /= p.n_kv_heads;
    const int block = id % p.s.suffix_blocks;
    id /= p.s.suffix_blocks;
    const int index = id % p.s.suffix_parts, seq = id / p.s.suffix_parts;
    const int begin = index * p.s.suffix_chunk, end = min(min(a.suffix_lens[seq], p.s.max_suffix), begin + p.s.suffix_chunk);
    if (begin >= end && !p.s.direct) return;
    part<T, kDim, 1, kMode>(p, a.suffix_pages + (int64_t)seq * a.suffix_width, begin, end, Members{seq, 1}, block * kRowsTile, kv_head,
                            p.s.prefix_parts + index, shared);
  }
}

// A wavefront to a row (sequence, query head): its parts in order, the prompt's first.
template <typename T, int kDim> __global__ __launch_bounds__(kThreads) void attend_merge(AttendParams p) {
  constexpr int kOwn = kDim / kWave;
  const hf_attention &a = p.a;
  const int lane = threadIdx.x % kWave;
  const int64_t row = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave;
  if (row >= (int64_t)a.n_seqs * a.n_q_heads) return;
  const int seq = row / a.n_q_heads, head = row % a.n_q_heads;
  int n_prefix = 0;
  for (int g0 = 0; g0 < a.n_groups; g0 += kWave) {
    const int g = g0 + lane;
    bool mine = false;
    if (g < a.n_groups) {
      const Members who = members(a, g);
      mine = seq >= who.first && seq < who.first + who.n;
    }
    const uint64_t found = __builtin_amdgcn_ballot_w64(mine);
    if (found) {
      const int len = min(a.prefix_lens[g0 + __builtin_ctzll(found)], p.s.max_prefix);
      n_prefix = len > 0 ? (len + p.s.prefix_chunk - 1) / p.s.prefix_chunk : 0;
      break;
    }
  }
  const int own = min(a.suffix_lens[seq], p.s.max_suffix), n_suffix = own > 0 ? (own + p.s.suffix_chunk - 1) / p.s.suffix_chunk : 0;
  const int n = n_prefix + n_suffix;
  const int64_t slot0 = row * (p.s.prefix_parts + p.s.suffix_parts);
  const auto slot = [&](int i) { return slot0 + (i < n_prefix ? i : p.s.prefix_parts + i - n_prefix); };
  float top = -INFINITY;
  for (int i = lane; i < n; i += kWave) top = fmaxf(top, p.part_ml[2 * slot(i)]);
#pragma unroll
  for (int d = kWave / 2; d; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
  float acc[kOwn] = {}, sum = 0;
#pragma unroll 4
  for (int i = 0; i < n; ++i) {
    const float m = p.part_ml[2 * slot(i)], l = p.part_ml[2 * slot(i) + 1];
    const float weight = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
    sum += weight * l;
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
      const int d = e * kWave + lane;
      if (d < p.head_dim) acc[e] += weight * p.part_o[slot(i) * p.head_dim + d];
    }
  }
  const float scale = sum == 0 ? 0.f : 1 / sum;
  T *to = static_cast<T *>(a.out) + seq * a.out_stride + head * a.out_head_stride;
#pragma unroll
  for (int e = 0; e < kOwn; ++e) {
    const int d = e * kWave + lane;
    if (d < p.head_dim) to[d] = (T)(acc[e] * scale);
  }
  if (a.lse && lane == 0) a.lse[row] = sum == 0 ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <typename T, int kDim, int kQ, int kMode> hipError_t launch_shape(const AttendParams &p, hipStream_t st) {
  const hipError_t e = enqueue_kernel(attend_parts<T, kDim, kQ, kMode>, dim3((uint32_t)(p.s.prefix_wgs + p.s.suffix_wgs)), kThreads, st, p);
  if (e != hipSuccess || p.s.direct) return e;
  const int64_t rows = (int64_t)p.a.n_seqs * p.a.n_q_heads;
  return enqueue_kernel(attend_merge<T, kDim>, dim3((uint32_t)((rows + kWaves - 1) / kWaves)), kThreads, st, p);
}
template <typename T, int kDim> hipError_t launch_dim(const AttendParams &p, bool vec, hipStream_t st) {
  const int mode = !vec ? kElements : p.head_dim == kDim ? kWhole : kPieces;
  if (mode == kElements) return launch_shape<T, kDim, 1, kElements>(p, st);
  if constexpr (kDim <= 128)
    if (p.s.q_tiles == 2) return mode == kWhole ? launch_shape<T, kDim, 2, kWhole>(p, st) : launch_shape<T, kDim, 2, kPieces>(p, st);
  return mode == kWhole ? launch_shape<T, kDim, 1, kWhole>(p, st) : launch_shape<T, kDim, 1, kPieces>(p, st);
}
template <typename T> hipError_t launch_type(const AttendParams &p, bool vec, hipStream_t st) {
  if (p.head_dim <= 64) return launch_dim<T, 64>(p, vec, st);
  if (p.head_dim <= 128) return launch_dim<T, 128>(p, vec, st);
  return launch_dim<T, 256>(p, vec, st);
}

} // namespace

AttendShape attend_shape(const hf_kv_cache &cache, const hf_attention &a, bool vec) {
  AttendShape s = {};
  const int64_t page = cache.page_tokens, ratio = a.n_q_heads / cache.n_kv_heads;
  s.max_suffix = (int32_t)std::min<int64_t>(a.max_suffix, std::min<int64_t>(a.suffix_width * page, 1 << 30));
  s.max_prefix = a.n_groups ? (int32_t)std::min<int64_t>(a.max_prefix, std::min<int64_t>(a.prefix_width * page, 1 << 30)) : 0;
  // parts: as long as they may be while there are about four workgroups a CU
  const auto chunk = [&](int64_t len, int64_t others) {
    int64_t c = 128;
    while (c < len && others * ((len + 2 * c - 1) / (2 * c)) >= 1024) c *= 2;
    return (int32_t)c;
  };
  const int64_t rows = std::min<int64_t>(a.max_group, a.n_seqs) * ratio;
  s.q_tiles = vec && cache.head_dim <= 128 && rows > kRowsTile ? 2 : 1;
  s.prefix_blocks = (int32_t)((rows + s.q_tiles * kRowsTile - 1) / (s.q_tiles * kRowsTile));
  s.suffix_blocks = (int32_t)((ratio + kRowsTile - 1) / kRowsTile);
  s.suffix_chunk = chunk(s.max_suffix, (int64_t)a.n_seqs * cache.n_kv_heads * s.suffix_blocks);
  s.prefix_chunk = chunk(s.max_prefix, (int64_t)a.n_groups * cache.n_kv_heads * s.prefix_blocks);
  s.suffix_parts = std::max(1, (s.max_suffix + s.suffix_chunk - 1) / s.suffix_chunk);
  s.prefix_parts = rows ? (s.max_prefix + s.prefix_chunk - 1) / s.prefix_chunk : 0;
  s.direct = s.prefix_parts == 0 && s.suffix_parts == 1;
  const uint64_t items = (uint64_t)a.n_groups * s.prefix_parts * cache.n_kv_heads;
  s.prefix_wgs = (items + 7) / 8 * 8 * s.prefix_blocks;
  s.suffix_wgs = (uint64_t)a.n_seqs * s.suffix_parts * s.suffix_blocks * cache.n_kv_heads;
  if (!s.direct) s.workspace = ((size_t)a.n_seqs * a.n_q_heads * (s.prefix_parts + s.suffix_parts)) * (cache.head_dim + 2) * sizeof(float);
  return s;
}

int launch_attend(const hf_kv_cache &cache, const hf_attention &a, const AttendShape &s, bool vec, void *stream) {
  AttendParams p = {a, s, cache.k, cache.v, cache.page_stride, cache.head_stride, cache.token_stride, (uint32_t)cache.n_pages,
                    cache.n_kv_heads, cache.head_dim, __builtin_ctz(cache.page_tokens), a.n_q_heads / cache.n_kv_heads, a.scale * kLog2e, nullptr, nullptr};
  if (!s.direct) {
    p.part_o = static_cast<float *>(a.workspace);
    p.part_ml = p.part_o + (size_t)a.n_seqs * a.n_q_heads * (s.prefix_parts + s.suffix_parts) * cache.head_dim;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  return (int)(cache.dtype == HF_BF16 ? launch_type<__bf16>(p, vec, st) : launch_type<_Float16>(p, vec, st));
}

} // namespace hf
