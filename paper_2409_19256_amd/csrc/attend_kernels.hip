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
//  - a wavefront takes tiles of 32 tokens straight from memory into registers, keys and values of the next tile on their way while it works on
//    the present one; nothing is staged and no wavefront waits for another until its part is done.  Where a prompt has many
//    rows the wavefronts of a workgroup take different rows over the same tokens and meet in the L1 cache;
//  - a page's number and address are the same for a whole wavefront and are worked out by the scalar unit (pages of 16 tokens and more);
//  - scores are made transposed, S^T = K Q^T: the accumulator then holds, for the query of a lane's column, four tokens of each 16, which
//    is what the second product O^T = V^T P^T wants as its right operand if its 32 tokens are taken in the order (16-token
//    half, lane group, token): P never moves between lanes;
//  - a lane loads 16 bytes of each of its eight tokens' values, whole rows over 16 lanes; the eight rows are turned in its registers (one byte
//    permute per two elements) into left operands for eight products, product j holding every eighth element of a head.
// Exponentials are of base 2, the scale carries the factor.  P is rounded to the cache's type twice, once for its upper bits and once for the
// rest: rounded once it would add as much to the error as the rounding of the output does.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "lanes.hpp"
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
template <typename T> __device__ __forceinline__ uint32_t load_two(const char *row, int d, int head_dim) {
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

// Rows row0 .. of a segment (the sequences [first, first + n), all of which see its tokens) over its tokens [begin, end).  kRowWaves wavefronts
// have kQ * 16 rows each, and the others the same rows over other tokens.
template <typename T, int kDim, int kQ, int kRowWaves, int kMode, bool kLanes>
__device__ __forceinline__ void part(const AttendParams &p, const int32_t *table, int begin, int end, Members who, int row0, int kv_head, int part_index,
                                     float *shared) {
  constexpr int kSteps = kDim / 32; // of the first product
  constexpr int kOwn = kDim / 16;   // elements of a value row that a lane holds, products of the second kind
  constexpr int kTokenWaves = kWaves / kRowWaves;
  const hf_attention &a = p.a;
  const int lane = threadIdx.x % kWave, col = lane % 16, grp = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), row_wave = wave % kRowWaves, token_wave = wave / kRowWaves;
  const int rows = who.n * p.ratio, my_row0 = row0 + row_wave * kQ * kRowsTile;
  const char *keys = p.k + kv_head * p.head_bytes, *values = p.v + kv_head * p.head_bytes;
  const int in_page = (1 << p.page_shift) - 1;

  u32x4 q[kQ][kSteps];
#pragma unroll
  for (int n = 0; n < kQ; ++n) {
    const int row = my_row0 + n * kRowsTile + col;
    const int seq = who.first + row / p.ratio, head = kv_head * p.ratio + row % p.ratio;
    const char *from = static_cast<const char *>(a.q) + (seq * a.q_stride + head * a.q_head_stride) * (int64_t)sizeof(T);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int d = 32 * s + 8 * grp;
      q[n][s] = u32x4{};
      if constexpr (kMode == kElements) {
        if (row < rows)
          for (int e = 0; e < 4; ++e) q[n][s][e] = load_two<T>(from, d + 2 * e, p.head_dim);
      } else if (row < rows && (kMode == kWhole || d < p.head_dim)) {
        q[n][s] = *reinterpret_cast<const u32x4 *>(from + 2 * d);
      }
      if (p.scale2 < 0) q[n][s] ^= 0x80008000u; // the maximum is taken of the products, so the scale has to be positive
    }
  }
  const float scale2 = fabsf(p.scale2);

  // Where a tile's tokens are.  A page of 16 tokens or more holds a half of a tile whole, so that its number is the same for all lanes and is
  // fetched and turned into an address by the scalar unit; with smaller pages every lane has its own.
  struct Pages {
    int k[2], v[2];
  };
  struct At {
    int64_t k[2], v[2]; // bytes from the head's first element
    bool ok[2];
  };
  const auto pages_at = [&](int token) {
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
  };
  // an unusable page number stands for page 0, whose tokens are then not seen
  const auto page_bytes = [&](int page) { return (int64_t)((uint32_t)page < p.n_pages ? (uint32_t)page : 0u) * p.page_bytes; };
  const auto place = [&](const Pages &g, int token) {
    At at;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      at.ok[h] = (uint32_t)g.v[h] < p.n_pages;
      if constexpr (kLanes) {
        at.k[h] = page_bytes(g.k[h]) + ((token + 16 * h + col) & in_page) * p.token_bytes + 16 * grp;
        at.v[h] = page_bytes(g.v[h]) + ((token + 16 * h + 4 * grp) & in_page) * p.token_bytes + 2 * kOwn * col;
      } else {
        at.k[h] = at.v[h] = page_bytes(g.k[h]) + ((token + 16 * h) & in_page) * p.token_bytes;
      }
    }
    return at;
  };
  // pieces past the head are read from its start, and left out when the result is written
  const uint32_t value_piece = kMode == kPieces && kOwn * col >= p.head_dim ? 0 : 2 * kOwn * col;
  const uint32_t k_lane = kLanes ? 0 : col * (uint32_t)p.token_bytes + 16 * grp;
  uint32_t v_lane[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v_lane[i] = kLanes ? 0 : (4 * grp + i) * (uint32_t)p.token_bytes + value_piece;

  const auto load_keys = [&](u32x4(&k)[2][kSteps], const At &at) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char *row = keys + at.k[h];
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int d = 32 * s + 8 * grp;
        if constexpr (kMode == kElements) {
          for (int e = 0; e < 4; ++e) k[h][s][e] = load_two<T>(row - 16 * grp, d + 2 * e, p.head_dim);
        } else if constexpr (kMode == kPieces) {
          k[h][s] = u32x4{};
          if (d < p.head_dim) k[h][s] = *reinterpret_cast<const u32x4 *>(row + k_lane + 64 * s);
        } else {
          k[h][s] = *reinterpret_cast<const u32x4 *>(row + k_lane + 64 * s);
        }
      }
    }
  };
  const auto load_values = [&](uint32_t(&v)[8][kOwn / 2], const At &at) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const char *row = kLanes ? values + at.v[h] + i * p.token_bytes : values + at.v[h] + v_lane[i];
        if constexpr (kMode == kElements) {
          for (int e = 0; e < kOwn / 2; ++e) v[4 * h + i][e] = load_two<T>(row - 2 * kOwn * col, kOwn * col + 2 * e, p.head_dim);
        } else {
          if constexpr (kLanes) row += (int)value_piece - 2 * kOwn * col;
          if constexpr (kOwn == 4) {
            const u32x2 x = *reinterpret_cast<const u32x2 *>(row);
            v[4 * h + i][0] = x[0], v[4 * h + i][1] = x[1];
          } else {
#pragma unroll
            for (int e = 0; e < kOwn / 8; ++e) { // the second piece of 16 elements may be past the head too
              const u32x4 x = *reinterpret_cast<const u32x4 *>(row + (kMode == kPieces && e && kOwn * col + 8 >= p.head_dim ? 0 : 16 * e));
#pragma unroll
              for (int f = 0; f < 4; ++f) v[4 * h + i][4 * e + f] = x[f];
            }
          }
        }
      }
    }
  };

  f32x4 o[kQ][kOwn];
  float m[kQ], l[kQ]; // m of the products, before the scale
#pragma unroll
  for (int n = 0; n < kQ; ++n) {
    m[n] = -INFINITY, l[n] = 0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) o[n][j] = f32x4{};
  }

  // Page numbers are fetched two tiles ahead.  The next tile's keys are on their way from when the scores are made, its values from when they are added
  // up: each is asked for as soon as its registers are free.
  constexpr int kStep = kTokenWaves * kTile;
  int token = begin + token_wave * kTile;
  if (token < end && my_row0 < rows) {
    u32x4 k[2][kSteps];
    uint32_t v[8][kOwn / 2];
    At at = place(pages_at(token), token);
    Pages next = pages_at(token + kStep);
    load_keys(k, at);
    load_values(v, at);
    for (;;) {
      const bool more = token + kStep < end;
      const bool whole = token + kTile <= end && (kLanes ? __builtin_amdgcn_ballot_w64(!(at.ok[0] && at.ok[1])) == 0 : at.ok[0] && at.ok[1]);
      bool seen[8];
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 8; ++i) seen[i] = at.ok[i / 4] && token + 16 * (i / 4) + 4 * grp + i % 4 < end;
      }
      f32x4 s[kQ][2];
#pragma unroll
      for (int n = 0; n < kQ; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          s[n][h] = f32x4{};
#pragma unroll
          for (int e = 0; e < kSteps; ++e) s[n][h] = Matrix<T>::product(k[h][e], q[n][e], s[n][h]);
        }
      at = place(next, token + kStep);
      if (more) {
        next = pages_at(token + 2 * kStep);
        load_keys(k, at);
      }
      u32x4 hi[kQ], lo[kQ];
#pragma unroll
      for (int n = 0; n < kQ; ++n) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = s[n][i / 4][i % 4];
        if (!whole) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = seen[i] ? x[i] : -INFINITY;
        }
        float top = x[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i]);
        const float m_new = fmaxf(m[n], over_rows<Max>(top));
        if (__builtin_amdgcn_ballot_w64(m_new > m[n]) != 0) {
          const float keep = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[n] - m_new) * scale2);
          m[n] = m_new;
          l[n] *= keep;
#pragma unroll
          for (int j = 0; j < kOwn; ++j) o[n][j] *= keep;
        }
        const float base = m[n] == -INFINITY ? 0.f : -m[n] * scale2;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], scale2, base));
        if (!whole) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = seen[i] ? x[i] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) l[n] += x[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          hi[n][i] = pack<T>(x[2 * i], x[2 * i + 1]);
          lo[n][i] = pack<T>(x[2 * i] - unpack<T>(hi[n][i], 0), x[2 * i + 1] - unpack<T>(hi[n][i], 1));
        }
      }
      if (!whole) { // what is not visible may hold anything, and 0 * NaN is no 0
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < kOwn / 2; ++e) v[i][e] = seen[i] ? v[i][e] : 0;
      }
#pragma unroll
      for (int j = 0; j < kOwn; ++j) {
        u32x4 left;
#pragma unroll
        for (int i = 0; i < 4; ++i) left[i] = __builtin_amdgcn_perm(v[2 * i + 1][j / 2], v[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int n = 0; n < kQ; ++n) o[n][j] = Matrix<T>::product(left, lo[n], Matrix<T>::product(left, hi[n], o[n][j]));
      }
      token += kStep;
      if (!more) break;
      load_values(v, at);
    }
  }

  // a row's sum and output, or its part of them
  const auto write = [&](int row, int d0, float top, float sum, const float *acc) {
    const int seq = who.first + row / p.ratio, head = kv_head * p.ratio + row % p.ratio;
    const int64_t at = (int64_t)seq * a.n_q_heads + head;
    const float m2 = top * scale2;
    if (p.s.direct) {
      const float scale = sum == 0 ? 0.f : 1 / sum;
      T *to = static_cast<T *>(a.out) + seq * a.out_stride + head * a.out_head_stride + d0;
#pragma unroll
      for (int e = 0; e < kOwn; ++e)
        if (kMode == kWhole || d0 + e < p.head_dim) to[e] = (T)(acc[e] * scale);
      if (a.lse && d0 == 0) a.lse[at] = sum == 0 ? -INFINITY : (m2 + __builtin_amdgcn_logf(sum)) * kLn2;
    } else {
      const int64_t slot = at * (p.s.prefix_parts + p.s.suffix_parts) + part_index;
      float *to = p.part_o + slot * p.head_dim + d0;
      if constexpr (kMode == kWhole) {
#pragma unroll
        for (int e = 0; e < kOwn; e += 4) *reinterpret_cast<f32x4 *>(to + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
      } else {
#pragma unroll
        for (int e = 0; e < kOwn; ++e)
          if (d0 + e < p.head_dim) to[e] = acc[e];
      }
      if (d0 == 0) p.part_ml[2 * slot] = top == -INFINITY ? -INFINITY : m2, p.part_ml[2 * slot + 1] = sum;
    }
  };

#pragma unroll
  for (int n = 0; n < kQ; ++n) l[n] = over_rows<Sum>(l[n]);
  if constexpr (kTokenWaves == 1) {
#pragma unroll
    for (int n = 0; n < kQ; ++n) {
      const int row = my_row0 + n * kRowsTile + col;
      if (row < rows) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float acc[kOwn];
#pragma unroll
          for (int j = 0; j < kOwn; ++j) acc[j] = o[n][j][i];
          write(row, kOwn * (4 * grp + i), m[n], l[n], acc);
        }
      }
    }
  } else { // the wavefronts' parts become one
    constexpr int kPitch = kDim + 4, kRows = kRowWaves * kRowsTile;
    float *const both = shared + kTokenWaves * kRows * kPitch; // [token wave, row, 2]
#pragma unroll
    for (int n = 0; n < kQ; ++n) {
      if (n) __syncthreads();
      const int mine = token_wave * kRows + row_wave * kRowsTile + col;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < kOwn; ++j) shared[mine * kPitch + kOwn * (4 * grp + i) + j] = o[n][j][i];
      if (grp == 0) both[2 * mine] = m[n], both[2 * mine + 1] = l[n];
      __syncthreads();
#pragma unroll
      for (int r0 = 0; r0 < kRows; r0 += kThreads / 16) {
        const int r = r0 + threadIdx.x / 16, d0 = threadIdx.x % 16 * kOwn;
        const int row = row0 + (r / kRowsTile * kQ + n) * kRowsTile + r % kRowsTile;
        if (row < rows) {
          float top = -INFINITY, sum = 0, acc[kOwn] = {};
#pragma unroll
          for (int w = 0; w < kTokenWaves; ++w) top = fmaxf(top, both[2 * (w * kRows + r)]);
#pragma unroll
          for (int w = 0; w < kTokenWaves; ++w) {
            const float mw = both[2 * (w * kRows + r)], weight = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mw - top) * scale2);
            sum += weight * both[2 * (w * kRows + r) + 1];
#pragma unroll
            for (int e = 0; e < kOwn; ++e) acc[e] += weight * shared[(w * kRows + r) * kPitch + d0 + e];
          }
          write(row, d0, top, sum, acc);
        }
      }
    }
  }
}

template <typename T, int kDim, int kQ, int kRowWaves, int kMode, bool kLanes>
__global__ __launch_bounds__(kThreads, kDim > 128 || kMode == kElements ? 1 : 2) void attend_parts(AttendParams p) {
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
    const int row0 = block * kRowWaves * kQ * kRowsTile;
    if (begin >= end || row0 >= who.n * p.ratio) return;
    part<T, kDim, kQ, kRowWaves, kMode, kLanes>(p, a.prefix_pages + (int64_t)g * a.prefix_width, begin, end, who, row0, kv_head, index, shared);
  } else {
    id -= p.s.prefix_wgs;
    const int kv_head = id % p.n_kv_heads;
    id /= p.n_kv_heads;
    const int block = id % p.s.suffix_blocks;
    id /= p.s.suffix_blocks;
    const int index = id % p.s.suffix_parts, seq = id / p.s.suffix_parts;
    const int begin = index * p.s.suffix_chunk, end = min(min(a.suffix_lens[seq], p.s.max_suffix), begin + p.s.suffix_chunk);
    if (begin >= end && !p.s.direct) return;
    part<T, kDim, 1, 1, kMode, kLanes>(p, a.suffix_pages + (int64_t)seq * a.suffix_width, begin, end, Members{seq, 1}, block * kRowsTile, kv_head,
                                       p.s.prefix_parts + index, shared);
  }
}

// A row (sequence, query head) out of its parts, in order.  kDim / 4 lanes have four elements of it each; `split` such teams share a row's parts
// where these are many, each taking every split-th.
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

template <typename T, int kDim, int kQ, int kRowWaves, int kMode, bool kLanes> hipError_t launch_shape(const AttendParams &p, hipStream_t st) {
  const hipError_t e = enqueue_kernel(attend_parts<T, kDim, kQ, kRowWaves, kMode, kLanes>, dim3((uint32_t)(p.s.prefix_wgs + p.s.suffix_wgs)), kThreads, st, p);
  if (e != hipSuccess || p.s.direct) return e;
  const int64_t rows = (int64_t)p.a.n_seqs * p.a.n_q_heads;
  constexpr int kTeams = kThreads / (kDim / 4);
  int split = 1;
  while (split < kTeams && 4 * split < p.s.prefix_parts + p.s.suffix_parts) split *= 2;
  const int rows_of_wg = kTeams / split;
  return enqueue_kernel(attend_merge<T, kDim>, dim3((uint32_t)((rows + rows_of_wg - 1) / rows_of_wg)), kThreads, st, p, split);
}
template <typename T, int kDim, int kMode, bool kLanes> hipError_t launch_rows(const AttendParams &p, hipStream_t st) {
  if constexpr (kDim <= 128 && kMode != kElements) {
    if (p.s.row_waves == 4) return launch_shape<T, kDim, 2, 4, kMode, kLanes>(p, st);
    if (p.s.row_waves == 2) return launch_shape<T, kDim, 2, 2, kMode, kLanes>(p, st);
    if (p.s.q_tiles == 2) return launch_shape<T, kDim, 2, 1, kMode, kLanes>(p, st);
  }
  return launch_shape<T, kDim, 1, 1, kMode, kLanes>(p, st);
}
template <typename T, int kDim> hipError_t launch_dim(const AttendParams &p, bool vec, hipStream_t st) {
  if (!vec) return launch_rows<T, kDim, kElements, true>(p, st);
  if (p.head_dim != kDim) return launch_rows<T, kDim, kPieces, true>(p, st);
  return p.s.lanes ? launch_rows<T, kDim, kWhole, true>(p, st) : launch_rows<T, kDim, kWhole, false>(p, st);
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
  // parts: as long as they may be while there are four workgroups a CU of responses, or one of prompts (whose parts cost every row a partial result:
  // us at 256 / 512 / 1024 workgroups, 128 samples of 8 prompts with 128 rows to a KV head 146 / 173 / 195, 61 samples of one of 32749 tokens with 488 62 / 72 / 87)
  const auto chunk = [&](int64_t len, int64_t others, int64_t want) {
    int64_t c = 128;
    while (c < len && others * ((len + 2 * c - 1) / (2 * c)) >= want) c *= 2;
    return (int32_t)c;
  };
  const int64_t rows = std::min<int64_t>(a.max_group, a.n_seqs) * ratio;
  s.q_tiles = vec && cache.head_dim <= 128 && rows > kRowsTile ? 2 : 1;
  s.row_waves = s.q_tiles == 1 || rows <= 2 * kRowsTile ? 1 : rows <= 4 * kRowsTile ? 2 : 4;
  s.lanes = page < 16 || cache.token_stride >= 1 << 25;
  const int64_t rows_of_wg = s.q_tiles * s.row_waves * kRowsTile;
  s.prefix_blocks = (int32_t)((rows + rows_of_wg - 1) / rows_of_wg);
  s.suffix_blocks = (int32_t)((ratio + kRowsTile - 1) / kRowsTile);
  s.suffix_chunk = chunk(s.max_suffix, (int64_t)a.n_seqs * cache.n_kv_heads * s.suffix_blocks, 1024);
  s.prefix_chunk = chunk(s.max_prefix, (int64_t)a.n_groups * cache.n_kv_heads * s.prefix_blocks, 256);
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
  AttendParams p = {a, s, static_cast<const char *>(cache.k), static_cast<const char *>(cache.v), 2 * cache.page_stride, 2 * cache.head_stride,
                    2 * cache.token_stride, (uint32_t)cache.n_pages,
                    cache.n_kv_heads, cache.head_dim, __builtin_ctz(cache.page_tokens), a.n_q_heads / cache.n_kv_heads, a.scale * kLog2e, nullptr, nullptr};
  if (!s.direct) {
    p.part_o = static_cast<float *>(a.workspace);
    p.part_ml = p.part_o + (size_t)a.n_seqs * a.n_q_heads * (s.prefix_parts + s.suffix_parts) * cache.head_dim;
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  return (int)(cache.dtype == HF_BF16 ? launch_type<__bf16>(p, vec, st) : launch_type<_Float16>(p, vec, st));
}

} // namespace hf
