// The pages of a model's caches: sequences that are dropped, go on or branch, room for new tokens, live pages moved to the lowest places.
//
// First the books, then the data.  The books are reference counts and page tables: counts are changed by atomics (whole numbers, in any order the same), and what has an
// order (the f-th free page to the f-th row that wants one) comes from sums over the rows and pages in front: of small batches by one workgroup with the counts in shared memory,
// else over tiles, each tile's own in one launch and everybody's in the next.  The books are bound by what follows one another (one workgroup 2.5-6 us, the launches 12-16).  The data are copied by the next
// launch, which HBM bounds: 8 accesses of 16 bytes of a lane in flight, stores past the caches, the parts of a page on one XCD.  us of copying: a fork of 32 sequences into 128 in 160 buffers, 251 MB
// written and, because three copies of a page are made by different workgroups, 182 read, 66-69 (6.4 TB/s); 245 pages of 512 KiB moved in four buffers, 1028 MB, 180 (5.7 TB/s).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "step_kernels.hpp"

namespace hf {

namespace {

constexpr int kThreads = 256, kWave = 64, kWaves = kThreads / kWave;
constexpr int kMostTiles = 1024; // whose sums a workgroup adds up by itself
constexpr int kPageTile = 1024, kRowTile = 256;

__host__ __device__ constexpr int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to; }
// items of a tile, a multiple of `least`
int64_t tile_of(int64_t n, int64_t least) { return least * std::max<int64_t>(1, up(up(n, kMostTiles), least)); }

// sums in front of every lane's x, and over the workgroup; `shared` holds one number a wavefront and may be used again at once
__device__ __forceinline__ int64_t sum_before(int64_t x, int64_t *shared, int64_t *all) {
  int64_t upto = x;
  for (int d = 1; d < kWave; d *= 2) {
    const int64_t y = __shfl_up((long long)upto, d);
    if ((int)threadIdx.x % kWave >= d) upto += y;
  }
  if (threadIdx.x % kWave == kWave - 1) shared[threadIdx.x / kWave] = upto;
  __syncthreads();
  int64_t base = 0, total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < (int)threadIdx.x / kWave) base += shared[w];
    total += shared[w];
  }
  __syncthreads();
  *all = total;
  return base + upto - x;
}
__device__ __forceinline__ int64_t sum_block(int64_t x, int64_t *shared) {
  int64_t all;
  sum_before(x, shared, &all);
  return all;
}
__device__ __forceinline__ int64_t sum_of(const int64_t *sums, int64_t n, int64_t *shared) {
  int64_t x = 0;
  for (int64_t i = threadIdx.x; i < n; i += kThreads) x += sums[i];
  return sum_block(x, shared);
}

// two numbers a lane, summed over the lanes in front and in all; for one use of `shared`
struct Pair {
  int32_t a, b;
};
template <int kControl, int kRows> __device__ __forceinline__ int32_t from_front(int32_t x) { return __builtin_amdgcn_update_dpp(0, x, kControl, kRows, 0xF, false); }
// with the lanes in front: 1, 2, 4 and 8 further in each row of 16, then the rows' ends
__device__ __forceinline__ int32_t row_sums(int32_t x) {
  x += from_front<0x111, 0xF>(x);
  x += from_front<0x112, 0xF>(x);
  x += from_front<0x114, 0xF>(x);
  return x + from_front<0x118, 0xF>(x);
}
__device__ __forceinline__ int32_t wave_sums(int32_t x) {
  x = row_sums(x);
  x += from_front<0x142, 0xA>(x);
  return x + from_front<0x143, 0xC>(x);
}
template <int kWaves> __device__ __forceinline__ Pair sums_before(Pair x, Pair (&shared)[kWaves], Pair *all) {
  static_assert(kWaves <= 16, "the wavefronts' sums lie in one row of lanes");
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const Pair upto = {wave_sums(x.a), wave_sums(x.b)};
  if (lane == kWave - 1) shared[wave] = upto;
  __syncthreads();
  const Pair theirs = lane < kWaves ? shared[lane] : Pair{0, 0}, sums = {row_sums(theirs.a), row_sums(theirs.b)};
  *all = {__builtin_amdgcn_readlane(sums.a, kWaves - 1), __builtin_amdgcn_readlane(sums.b, kWaves - 1)};
  const Pair base = {wave ? __builtin_amdgcn_readlane(sums.a, wave - 1) : 0, wave ? __builtin_amdgcn_readlane(sums.b, wave - 1) : 0};
  return {base.a + upto.a - x.a, base.b + upto.b - x.b};
}
// a lane's pages of an array, four at a time: loaded as far as they go, the others are `none`
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_any __attribute__((aligned(4)));
__device__ __forceinline__ i32x4 four_of(const int32_t *from, int64_t i, int64_t n, int32_t none) {
  if (i + 4 <= n) return *reinterpret_cast<const i32x4_any *>(from + i);
  i32x4 v = none;
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (i + e < n) v[e] = from[i + e];
  return v;
}

// Tables of page numbers, and what of a row counts.
struct Tables {
  const int32_t *entries, *lens;
  int32_t rows, width, shift; // page_tokens = 2^shift
  int32_t n_pages;
};
__device__ __forceinline__ int64_t len_of(const Tables &t, int64_t row) { return min((int64_t)max(t.lens[row], 0), (int64_t)t.width << t.shift); }
__device__ __forceinline__ int64_t pages_of(const Tables &t, int64_t len) { return (len + (1 << t.shift) - 1) >> t.shift; }
__device__ __forceinline__ int32_t page_at(const Tables &t, int64_t row, int64_t i) {
  const int32_t p = t.entries[row * t.width + i];
  return p >= 0 && p < t.n_pages ? p : -1;
}

// ---- the data ------------------------------------------------------------------------------------------------------------

// How the tokens of a page lie in a cache, in elements: runs of `inner`, of which there are outer * middle.  One of the three grows with the number of tokens.
struct Shape {
  int64_t page, outer_stride, middle_stride;
  int32_t outer, middle, inner;
  int32_t growing; // 0: outer, 1: middle, 2: inner
};
struct Buffers {
  void *at[2 * HF_MAX_CACHES];
  int32_t n;
};

// A run of at least 8 elements is copied 8 at a time wherever it begins, the last ones of it ending where it ends: what two of them have in common is written twice, alike.
// Three heads of 65 in pages of 32, half of 1580 pages live, five layers: 22.9 us where single elements took 52.6; heads of 72 and 128 level with accesses that know their alignment.
template <int kVec> struct Access {
  typedef uint16_t type __attribute__((ext_vector_type(kVec)));
  typedef type any __attribute__((aligned(2)));
};
template <> struct Access<1> {
  typedef uint16_t type, any;
};

// us of fork / compact as above, with plain loads and non-temporal stores: 4 in flight 79 / 203, 8 70 / 205; plain stores 103 / 212 (4).  Loads past the caches: 125 / 196 (4), so that
// compact, whose pages are read once, has them and fork does not.
constexpr int kInFlight = 8;

// Accesses [part * kThreads * kInFlight, ...) of the first `tokens` tokens of a page, on their way from one to others.  kOnce: read past the caches.
template <int kVec, bool kOnce> struct Part {
  typedef typename Access<kVec>::any V;
  int64_t off[kInFlight];
  typename Access<kVec>::type v[kInFlight];
  uint32_t at0, n;
  __device__ __forceinline__ void load(const void *buffer, const Shape &s, int64_t page, int32_t tokens, uint32_t part) {
    const uint32_t outer = s.growing == 0 ? tokens : s.outer, middle = s.growing == 1 ? tokens : s.middle, inner = s.growing == 2 ? s.inner * tokens : s.inner;
    const uint32_t each = (inner + kVec - 1) / kVec;
    n = outer * middle * each; // (fits: a page has fewer than 2^31 elements)
    at0 = part * (kThreads * kInFlight) + threadIdx.x;
    const uint16_t *base = static_cast<const uint16_t *>(buffer) + page * s.page;
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      const uint32_t at = at0 + k * kThreads;
      if (at >= n) break;
      const uint32_t run = at / each, x = min(at % each * kVec, inner - kVec);
      off[k] = s.growing == 1 ? run / middle * s.outer_stride + run % middle * s.middle_stride + x : run * s.outer_stride + x;
      const V *from = reinterpret_cast<const V *>(base + off[k]);
      v[k] = kOnce ? __builtin_nontemporal_load(from) : *from;
    }
  }
  __device__ __forceinline__ void store(void *buffer, const Shape &s, int64_t page) const {
    uint16_t *base = static_cast<uint16_t *>(buffer) + page * s.page;
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      if (at0 + k * kThreads >= n) break;
      __builtin_nontemporal_store(v[k], reinterpret_cast<V *>(base + off[k]));
    }
  }
};

// What moves: the first `tokens` tokens of a page, to another one.
struct Move {
  int32_t from, tokens;
};
// Moves dealt out by parts of a page: f(move, buffer, part) for every `wgs`-th, from `wg` on.  The parts of a page go to one XCD (workgroups go round them by eights):
// 1024 pages of 512 KiB in four buffers, 245 of them moved, 187 us for 205.
template <typename F> __device__ __forceinline__ void each_part(int64_t moves, uint32_t buffers, uint32_t parts, uint32_t wg, uint32_t wgs, const F &f) {
  const uint32_t turn = 8 * parts;
  if (wg < wgs / turn * turn) wg = wg / turn * turn + wg % 8 * parts + wg % turn / 8;
  const uint32_t per = buffers * parts, step = wgs / per, more = wgs % per;
  int64_t k = wg / per;
  for (uint32_t i = wg % per; k < moves; k += step, i += more) {
    if (i >= per) {
      i -= per;
      if (++k >= moves) break;
    }
    f(k, i / parts, i % parts);
  }
}

// ---- fork ----------------------------------------------------------------------------------------------------------------

struct Fork {
  Tables from;
  const int32_t *parents, *refs;
  int32_t *tables_out, *lens_out, *refs_out;
  int32_t rows_out;
  // workspace
  int32_t *first;            // [n_pages] the first row that goes on in a page that is not full
  int64_t *free_sums, *want_sums; // per tile of pages, of rows
  int32_t *free_list;        // [rows_out]
  int32_t *want;             // [rows_out] which free page a row wants; -1 none
  Move *moves;               // [rows_out] what goes into those that are wanted
  int64_t *totals;           // free pages, wanted pages
  int32_t page_tiles, row_tiles;
  int64_t page_tile, row_tile;
};
__device__ __forceinline__ int64_t parent_of(const Fork &f, int64_t row) {
  const int32_t p = f.parents[row];
  return p >= 0 && p < f.from.rows ? p : -1;
}
// the page that a row goes on in, if it is not full: else -1
__device__ __forceinline__ int32_t open_page(const Fork &f, int64_t parent) {
  if (parent < 0) return -1;
  const int64_t len = len_of(f.from, parent);
  return len & ((1 << f.from.shift) - 1) ? page_at(f.from, parent, len >> f.from.shift) : -1;
}
__device__ __forceinline__ bool is_free(const Fork &f, int64_t page) { return f.refs_out[page] == 0 && f.first[page] == INT32_MAX; }

__global__ __launch_bounds__(kThreads) void fork_begin(Fork f) {
  for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < f.from.n_pages; i += (int64_t)gridDim.x * kThreads) {
    if (f.refs_out != f.refs) f.refs_out[i] = f.refs[i];
    f.first[i] = INT32_MAX;
  }
}
// a wavefront to a row: old rows give their pages back, new ones take theirs
__global__ __launch_bounds__(kThreads) void fork_count(Fork f) {
  const int lane = threadIdx.x % kWave;
  for (int64_t i = blockIdx.x * (int64_t)kWaves + threadIdx.x / kWave; i < (int64_t)f.from.rows + f.rows_out; i += (int64_t)gridDim.x * kWaves) {
    const bool old = i < f.from.rows;
    const int64_t r = old ? i : i - f.from.rows, row = old ? r : parent_of(f, r);
    if (row < 0) continue;
    const int64_t len = len_of(f.from, row), n = old ? pages_of(f.from, len) : len >> f.from.shift;
    for (int64_t k = lane; k < n; k += kWave)
      if (const int32_t p = page_at(f.from, row, k); p >= 0) atomicAdd(&f.refs_out[p], old ? -1 : 1);
    if (!old && lane == 0)
      if (const int32_t p = open_page(f, row); p >= 0) atomicMin(&f.first[p], (int32_t)r);
  }
}
__global__ __launch_bounds__(kThreads) void fork_sums(Fork f) {
  __shared__ int64_t shared[kWaves];
  int64_t n = 0;
  if ((int)blockIdx.x < f.page_tiles) {
    const int64_t begin = blockIdx.x * f.page_tile, end = min(begin + f.page_tile, (int64_t)f.from.n_pages);
    for (int64_t i = begin + threadIdx.x; i < end; i += kThreads) n += is_free(f, i);
    n = sum_block(n, shared);
    if (threadIdx.x == 0) f.free_sums[blockIdx.x] = n;
  } else {
    const int64_t tile = blockIdx.x - f.page_tiles, begin = tile * f.row_tile, end = min(begin + f.row_tile, (int64_t)f.rows_out);
    for (int64_t r = begin + threadIdx.x; r < end; r += kThreads) {
      const int32_t p = open_page(f, parent_of(f, r));
      n += p >= 0 && f.first[p] != r;
    }
    n = sum_block(n, shared);
    if (threadIdx.x == 0) f.want_sums[tile] = n;
  }
}
__global__ __launch_bounds__(kThreads) void fork_lists(Fork f) {
  __shared__ int64_t shared[kWaves];
  __shared__ Pair pairs[kWaves];
  int64_t all;
  if ((int)blockIdx.x < f.page_tiles) {
    int32_t base = (int32_t)sum_of(f.free_sums, blockIdx.x, shared);
    const int64_t begin = blockIdx.x * f.page_tile, end = min(begin + f.page_tile, (int64_t)f.from.n_pages);
    for (int64_t i0 = begin; i0 < end; i0 += 4 * kThreads) {
      const int64_t i = i0 + 4 * threadIdx.x;
      const i32x4 refs = four_of(f.refs_out, i, end, 1), first = four_of(f.first, i, end, INT32_MAX);
      Pair mine = {0, 0}, sums;
#pragma unroll
      for (int e = 0; e < 4; ++e) mine.a += refs[e] == 0 && first[e] == INT32_MAX;
      int32_t at = base + sums_before(mine, pairs, &sums).a;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (first[e] != INT32_MAX) f.refs_out[i + e] = refs[e] + 1;
        else if (refs[e] == 0 && at++ < f.rows_out) f.free_list[at - 1] = (int32_t)(i + e);
      }
      base += sums.a;
      __syncthreads();
    }
    if ((int)blockIdx.x == f.page_tiles - 1 && threadIdx.x == 0) f.totals[0] = base;
  } else {
    const int64_t tile = blockIdx.x - f.page_tiles, begin = tile * f.row_tile, end = min(begin + f.row_tile, (int64_t)f.rows_out);
    int64_t base = sum_of(f.want_sums, tile, shared);
    for (int64_t r0 = begin; r0 < end; r0 += kThreads) {
      const int64_t r = r0 + threadIdx.x;
      const int32_t p = r < end ? open_page(f, parent_of(f, r)) : -1;
      const bool wants = p >= 0 && f.first[p] != r;
      const int64_t at = base + sum_before(wants, shared, &all);
      if (r < end) f.want[r] = wants ? (int32_t)at : -1;
      if (wants) f.moves[at] = {p, (int32_t)(len_of(f.from, parent_of(f, r)) & ((1 << f.from.shift) - 1))};
      base += all;
    }
    if (tile == f.row_tiles - 1 && threadIdx.x == 0) f.totals[1] = base;
  }
}
// what a place of a new row's table holds; `refs`: the counts, in memory or shared
__device__ __forceinline__ int32_t forked(const Fork &f, int32_t *refs, int64_t parent, int64_t n, int64_t k, bool lost, int32_t fresh) {
  int32_t p = k < n ? page_at(f.from, parent, k) : -1;
  if (lost) {
    if (p >= 0 && k < n - 1) atomicAdd(&refs[p], -1);
    return -1;
  }
  if (fresh >= 0 && k == n - 1) refs[p = fresh] = 1;
  return p;
}
__device__ __forceinline__ void fork_rows(const Fork &f, int64_t wave, int64_t waves) {
  const int64_t free = f.totals[0];
  for (int64_t r = wave; r < f.rows_out; r += waves) {
    const int64_t parent = parent_of(f, r), len = parent < 0 ? 0 : len_of(f.from, parent), n = pages_of(f.from, len);
    const int32_t want = f.want[r];
    const bool lost = want >= free;
    const int32_t fresh = want >= 0 && !lost ? f.free_list[want] : -1;
    for (int64_t k = threadIdx.x % kWave; k < f.from.width; k += kWave) f.tables_out[r * f.from.width + k] = forked(f, f.refs_out, parent, n, k, lost, fresh);
    if (threadIdx.x % kWave == 0) f.lens_out[r] = lost ? 0 : (int32_t)len;
  }
}
// Moves of a fork that a workgroup takes together.  us at 1 / 2 / 4 / 8: 16 prompts of up to 1000 tokens, 64 samples each in order, 32 layers of 8 heads (6.9 GB) 1940 / 1470 / 1288 / 1299, samples in
// any order 1720 / 1720 / 1702 / 1726; 32 sequences into 128 in 160 buffers, in order, 57 / 59 / 61 / 63: as many moves as there are workgroups have nothing to gain.
constexpr int kTogether = 4;
// row_wgs: workgroups that write tables, a wavefront to a row; the others copy
template <int kVec> __global__ __launch_bounds__(kThreads) void fork_apply(Fork f, Buffers buffers, Shape shape, uint32_t row_wgs, uint32_t parts) {
  if (blockIdx.x < row_wgs) return fork_rows(f, blockIdx.x * (int64_t)kWaves + threadIdx.x / kWave, (int64_t)row_wgs * kWaves);
  const int64_t moves = min(f.totals[0], f.totals[1]);
  // Where there is enough to do, moves that follow one another are taken together, and read once if they are of one page (a prompt that goes on as many samples).
  const int64_t together = moves * buffers.n * parts >= (int64_t)kTogether * (gridDim.x - row_wgs) ? kTogether : 1;
  each_part((moves + together - 1) / together, buffers.n, parts, blockIdx.x - row_wgs, gridDim.x - row_wgs, [&](int64_t group, uint32_t b, uint32_t part) {
    Part<kVec, false> data;
    Move had = {-1, 0};
    for (int64_t k = group * together; k < min(moves, (group + 1) * together); ++k) {
      const Move m = f.moves[k];
      if (m.from != had.from || m.tokens != had.tokens) data.load(buffers.at[b], shape, m.from, m.tokens, part);
      had = m;
      data.store(buffers.at[b], shape, f.free_list[k]);
    }
  });
}

// All of the books by one workgroup, counts in shared memory.
constexpr int kSoloThreads = 1024, kSoloWaves = kSoloThreads / kWave, kSoloPages = 8192, kSoloRows = 2048;
constexpr int kSoloEach = kSoloPages / kSoloThreads; // pages of a lane, one after another
__device__ __forceinline__ int each_of(int pages) { return (pages + 4 * kSoloThreads - 1) / (4 * kSoloThreads) * 4; } // of a lane, a multiple of four

__global__ __launch_bounds__(kSoloThreads) void fork_solo(Fork f) {
  __shared__ __attribute__((aligned(16))) int32_t refs[kSoloPages], first[kSoloPages];
  __shared__ int32_t lens[kSoloRows], parents[kSoloRows];
  __shared__ Pair shared[kSoloWaves];
  const int t = threadIdx.x, width = f.from.width, pages = f.from.n_pages, part = (1 << f.from.shift) - 1;
#pragma unroll 4
  for (int i = t; i < pages; i += kSoloThreads) refs[i] = f.refs[i], first[i] = INT32_MAX;
  for (int r = t; r < f.from.rows; r += kSoloThreads) lens[r] = (int32_t)len_of(f.from, r);
  for (int r = t; r < f.rows_out; r += kSoloThreads) parents[r] = (int32_t)parent_of(f, r);
  __syncthreads();
  const auto len_at = [&](int parent) { return parent < 0 ? 0 : lens[parent]; };
  const auto open_at = [&](int parent) { return len_at(parent) & part ? page_at(f.from, parent, lens[parent] >> f.from.shift) : -1; };
#pragma unroll 4
  for (int i = t; i < f.from.rows * width; i += kSoloThreads) {
    const int r = i / width, k = i % width;
    if (k < pages_of(f.from, lens[r]))
      if (const int32_t p = page_at(f.from, r, k); p >= 0) atomicAdd(&refs[p], -1);
  }
#pragma unroll 4
  for (int i = t; i < f.rows_out * width; i += kSoloThreads) {
    const int r = i / width, k = i % width, parent = parents[r], len = len_at(parent), full = len >> f.from.shift;
    if (k < pages_of(f.from, len))
      if (const int32_t p = page_at(f.from, parent, k); p >= 0) {
        if (k < full) atomicAdd(&refs[p], 1);
        else atomicMin(&first[p], r);
      }
  }
  // a lane's rows and pages lie one after another: what stands in front of them is one sum
  constexpr int kRows = kSoloRows / kSoloThreads;
  const int rows_each = (f.rows_out + kSoloThreads - 1) / kSoloThreads;
  int32_t open[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int r = t * rows_each + k;
    open[k] = k < rows_each && r < f.rows_out ? open_at(parents[r]) : -1;
  }
  __syncthreads();
  Pair mine = {0, 0}, all;
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    if (open[k] >= 0 && first[open[k]] == t * rows_each + k) open[k] = -1;
    mine.a += open[k] >= 0;
  }
  const int each = each_of(pages);
  uint32_t is_free = 0;
#pragma unroll
  for (int k = 0; k < kSoloEach; k += 4) {
    const int i = t * each + k;
    if (k >= each || i >= pages) break;
    const i32x4 n = *reinterpret_cast<const i32x4 *>(refs + i), held = *reinterpret_cast<const i32x4 *>(first + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (i + e >= pages) continue;
      if (held[e] != INT32_MAX) refs[i + e] = n[e] + 1; // the first row that goes on in it has it
      else if (n[e] == 0) is_free |= 1u << (k + e);
    }
  }
  mine.b = __popc(is_free);
  Pair at = sums_before(mine, shared, &all);
  const int32_t wanted = all.a, free = all.b;
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int r = t * rows_each + k;
    if (k >= rows_each || r >= f.rows_out) continue;
    f.want[r] = open[k] >= 0 ? at.a : -1;
    if (open[k] >= 0) f.moves[at.a++] = {open[k], len_at(parents[r]) & part};
  }
  for (uint32_t left = is_free; left; left &= left - 1, ++at.b)
    if (at.b < wanted) f.free_list[at.b] = t * each + __builtin_ctz(left);
  if (t == 0) f.totals[0] = free, f.totals[1] = wanted;
  __syncthreads();
#pragma unroll 4
  for (int i = t; i < f.rows_out * width; i += kSoloThreads) {
    const int r = i / width, k = i % width, parent = parents[r];
    const int32_t want = f.want[r];
    const bool lost = want >= free;
    f.tables_out[i] = forked(f, refs, parent, pages_of(f.from, len_at(parent)), k, lost, want >= 0 && !lost ? f.free_list[want] : -1);
  }
  for (int r = t; r < f.rows_out; r += kSoloThreads) f.lens_out[r] = f.want[r] >= free ? 0 : len_at(parents[r]);
  __syncthreads();
  for (int i = t; i < pages; i += kSoloThreads) f.refs_out[i] = refs[i];
}

// ---- grow ----------------------------------------------------------------------------------------------------------------

struct Grow {
  Tables from;
  const int32_t *counts, *refs;
  int32_t *tables_out, *lens_out, *refs_out;
  int64_t *slots;
  int32_t most;
  // workspace
  int64_t *free_sums, *want_sums, *before; // before [rows]: pages that the rows in front want
  int32_t *free_list;
  int64_t *totals;
  int64_t list; // most free pages that can be wanted
  int32_t page_tiles, row_tiles;
  int64_t page_tile, row_tile;
};
struct Growth {
  int64_t len, have, want; // tokens, pages, pages wanted in all
  int32_t count;
  bool fits;
  __device__ int64_t need() const { return fits ? want - have : 0; }
};
__device__ __forceinline__ Growth growth_of(const Grow &g, int64_t row) {
  Growth x;
  x.len = len_of(g.from, row), x.have = pages_of(g.from, x.len);
  x.count = min(max(g.counts[row], 0), g.most);
  x.want = pages_of(g.from, x.len + x.count);
  x.fits = x.want <= g.from.width && x.len + x.count <= INT32_MAX;
  return x;
}

__global__ __launch_bounds__(kThreads) void grow_sums(Grow g) {
  __shared__ int64_t shared[kWaves];
  int64_t n = 0;
  if ((int)blockIdx.x < g.page_tiles) {
    const int64_t begin = blockIdx.x * g.page_tile, end = min(begin + g.page_tile, (int64_t)g.from.n_pages);
    for (int64_t i = begin + threadIdx.x; i < end; i += kThreads) {
      const int32_t refs = g.refs[i];
      n += refs == 0;
      if (g.refs_out != g.refs) g.refs_out[i] = refs;
    }
    n = sum_block(n, shared);
    if (threadIdx.x == 0) g.free_sums[blockIdx.x] = n;
  } else {
    const int64_t tile = blockIdx.x - g.page_tiles, begin = tile * g.row_tile, end = min(begin + g.row_tile, (int64_t)g.from.rows);
    for (int64_t r = begin + threadIdx.x; r < end; r += kThreads) n += growth_of(g, r).need();
    n = sum_block(n, shared);
    if (threadIdx.x == 0) g.want_sums[tile] = n;
  }
}
__global__ __launch_bounds__(kThreads) void grow_lists(Grow g) {
  __shared__ int64_t shared[kWaves];
  __shared__ Pair pairs[kWaves];
  int64_t all;
  if ((int)blockIdx.x < g.page_tiles) {
    const int64_t begin = blockIdx.x * g.page_tile, end = min(begin + g.page_tile, (int64_t)g.from.n_pages);
    i32x4 refs = four_of(g.refs_out, begin + 4 * threadIdx.x, end, 1);
    int32_t base = (int32_t)sum_of(g.free_sums, blockIdx.x, shared);
    for (int64_t i0 = begin; i0 < end; i0 += 4 * kThreads) {
      const int64_t i = i0 + 4 * threadIdx.x;
      if (i0 > begin) refs = four_of(g.refs_out, i, end, 1);
      Pair mine = {0, 0}, sums;
#pragma unroll
      for (int e = 0; e < 4; ++e) mine.a += refs[e] == 0;
      int32_t at = base + sums_before(mine, pairs, &sums).a;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (refs[e] == 0 && at++ < g.list) g.free_list[at - 1] = (int32_t)(i + e);
      base += sums.a;
      __syncthreads();
    }
    if ((int)blockIdx.x == g.page_tiles - 1 && threadIdx.x == 0) g.totals[0] = base;
  } else {
    const int64_t tile = blockIdx.x - g.page_tiles, begin = tile * g.row_tile, end = min(begin + g.row_tile, (int64_t)g.from.rows);
    int64_t base = sum_of(g.want_sums, tile, shared);
    for (int64_t r0 = begin; r0 < end; r0 += kThreads) {
      const int64_t r = r0 + threadIdx.x;
      const int64_t at = base + sum_before(r < end ? growth_of(g, r).need() : 0, shared, &all);
      if (r < end) g.before[r] = at;
      base += all;
    }
  }
}
// a wavefront to a row
__global__ __launch_bounds__(kThreads) void grow_apply(Grow g) {
  const int lane = threadIdx.x % kWave, page_tokens = 1 << g.from.shift;
  const int64_t free = g.totals[0];
  for (int64_t r = blockIdx.x * (int64_t)kWaves + threadIdx.x / kWave; r < g.from.rows; r += (int64_t)gridDim.x * kWaves) {
    const Growth x = growth_of(g, r);
    const int64_t before = g.before[r];
    const bool ok = x.fits && (x.need() == 0 || before + x.need() <= free);
    const int32_t open = x.len % page_tokens ? page_at(g.from, r, x.have - 1) : -1; // the page that the first new tokens go to
    for (int64_t k = lane; k < g.from.width; k += kWave) {
      int32_t p = k < x.have ? page_at(g.from, r, k) : -1;
      if (ok && k >= x.have && k < x.want) {
        p = g.free_list[before + k - x.have];
        g.refs_out[p] = 1;
      }
      g.tables_out[r * g.from.width + k] = p;
    }
    for (int64_t i = lane; i < g.most; i += kWave) {
      const int64_t at = x.len + i, k = at >> g.from.shift;
      int64_t slot = -1;
      if (ok && i < x.count) {
        const int64_t p = k < x.have ? open : g.free_list[before + k - x.have];
        if (p >= 0) slot = (p << g.from.shift) + (at & (page_tokens - 1));
      }
      __builtin_nontemporal_store(slot, g.slots + r * g.most + i); // (plain stores: 4096 rows of 1024 in 17.9 us for 15.7)
    }
    if (lane == 0) g.lens_out[r] = (int32_t)(ok ? x.len + x.count : x.len);
  }
}

// All of it by one workgroup.
constexpr int kSoloFresh = 8192; // fresh pages that it can hand out
__global__ __launch_bounds__(kSoloThreads) void grow_solo(Grow g) {
  __shared__ int32_t list[kSoloFresh], before[kSoloRows], lens[kSoloRows], counts[kSoloRows];
  __shared__ Pair shared[kSoloWaves];
  const int t = threadIdx.x, width = g.from.width, pages = g.from.n_pages, shift = g.from.shift, page_tokens = 1 << shift;
  // a lane's rows and pages lie one after another: what stands in front of them is one sum
  const int each = each_of(pages), rows_each = (g.from.rows + kSoloThreads - 1) / kSoloThreads;
  i32x4 refs[kSoloEach / 4];
#pragma unroll
  for (int k = 0; k < kSoloEach; k += 4)
    if (k < each) refs[k / 4] = four_of(g.refs, t * each + k, pages, 1);
  constexpr int kRows = kSoloRows / kSoloThreads;
  int32_t need[kRows];
  Pair mine = {0, 0}, all;
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int r = t * rows_each + k;
    need[k] = 0;
    if (k >= rows_each || r >= g.from.rows) continue;
    const Growth x = growth_of(g, r);
    need[k] = (int32_t)x.need();
    lens[r] = (int32_t)x.len, counts[r] = x.fits ? x.count : -1;
    mine.a += need[k];
  }
  uint32_t is_free = 0;
#pragma unroll
  for (int k = 0; k < kSoloEach; ++k)
    if (k < each && refs[k / 4][k % 4] == 0) is_free |= 1u << k;
  mine.b = __popc(is_free);
  Pair at = sums_before(mine, shared, &all);
  const int32_t wanted = all.a, free = all.b;
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int r = t * rows_each + k;
    if (k < rows_each && r < g.from.rows) before[r] = at.a, at.a += need[k];
  }
  for (uint32_t left = is_free; left; left &= left - 1, ++at.b)
    if (at.b < wanted) list[at.b] = t * each + __builtin_ctz(left);
  if (g.refs_out != g.refs) {
#pragma unroll
    for (int k = 0; k < kSoloEach; ++k)
      if (const int i = t * each + k; k < each && i < pages) g.refs_out[i] = refs[k / 4][k % 4];
  }
  __syncthreads();
  const auto grows = [&](int r, int32_t &have, int32_t &want) {
    have = (int32_t)pages_of(g.from, lens[r]), want = (int32_t)pages_of(g.from, lens[r] + (int64_t)max(counts[r], 0));
    return counts[r] >= 0 && (want == have || before[r] + want - have <= free);
  };
  int32_t have, want;
#pragma unroll 2
  for (int i = t; i < g.from.rows * g.most; i += kSoloThreads) { // (the tables are read before they are written: they may be the same)
    const int r = i / g.most;
    const int64_t at = (int64_t)lens[r] + i % g.most, k = at >> shift;
    int64_t slot = -1;
    if (grows(r, have, want) && i % g.most < counts[r]) {
      const int64_t p = k < have ? page_at(g.from, r, k) : list[before[r] + k - have];
      if (p >= 0) slot = (p << shift) + (at & (page_tokens - 1));
    }
    g.slots[i] = slot;
  }
  __syncthreads();
#pragma unroll 4
  for (int i = t; i < g.from.rows * width; i += kSoloThreads) {
    const int r = i / width, k = i % width;
    const bool ok = grows(r, have, want);
    int32_t p = k < have ? page_at(g.from, r, k) : -1;
    if (ok && k >= have && k < want) g.refs_out[p = list[before[r] + k - have]] = 1;
    g.tables_out[i] = p;
  }
  for (int r = t; r < g.from.rows; r += kSoloThreads) g.lens_out[r] = lens[r] + (grows(r, have, want) ? counts[r] : 0);
}

// ---- compact -------------------------------------------------------------------------------------------------------------

struct Compact {
  const int32_t *refs;
  int32_t *refs_out, *places, *live;
  const int32_t *entries[HF_MAX_TABLES];
  int32_t *entries_out[HF_MAX_TABLES];
  int64_t n_entries[HF_MAX_TABLES];
  // workspace
  int64_t *live_sums;
  int32_t *from, *to; // [n_pages / 2]
  int64_t *totals;    // pairs
  int32_t n_pages, page_tiles;
  int64_t page_tile;
};

__global__ __launch_bounds__(kThreads) void compact_sums(Compact c) {
  __shared__ int64_t shared[kWaves];
  const int64_t begin = blockIdx.x * c.page_tile, end = min(begin + c.page_tile, (int64_t)c.n_pages);
  int64_t n = 0;
  for (int64_t i = begin + threadIdx.x; i < end; i += kThreads) n += c.refs[i] != 0;
  n = sum_block(n, shared);
  if (threadIdx.x == 0) c.live_sums[blockIdx.x] = n;
}
__global__ __launch_bounds__(kThreads) void compact_lists(Compact c) {
  __shared__ int64_t shared[kWaves];
  __shared__ Pair pairs[kWaves];
  const int64_t live = sum_of(c.live_sums, c.page_tiles, shared);
  // those in use below number `live`, which stay
  const int64_t whole = live / c.page_tile;
  int64_t stay = 0;
  for (int64_t i = whole * c.page_tile + threadIdx.x; i < live; i += kThreads) stay += c.refs[i] != 0;
  stay = sum_block(stay, shared) + sum_of(c.live_sums, whole, shared);
  int32_t base = (int32_t)sum_of(c.live_sums, blockIdx.x, shared);
  const int64_t begin = blockIdx.x * c.page_tile, end = min(begin + c.page_tile, (int64_t)c.n_pages);
  for (int64_t i0 = begin; i0 < end; i0 += 4 * kThreads) {
    const int64_t i = i0 + 4 * threadIdx.x;
    const i32x4 refs = four_of(c.refs, i, end, 0);
    Pair mine = {0, 0}, sums;
#pragma unroll
    for (int e = 0; e < 4; ++e) mine.a += refs[e] != 0;
    int32_t before = base + sums_before(mine, pairs, &sums).a; // in use in front of a page
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (i + e >= end) continue;
      const bool is = refs[e] != 0;
      if (is && i + e >= live) c.from[before - stay] = (int32_t)(i + e);
      if (!is && i + e < live) c.to[i + e - before] = (int32_t)(i + e);
      c.places[i + e] = is && i + e < live ? (int32_t)(i + e) : -1;
      before += is;
    }
    base += sums.a;
    __syncthreads();
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) c.totals[0] = live - stay, *c.live = (int32_t)live;
}
// the counts of pages that stay, and those that move with theirs
__global__ __launch_bounds__(kThreads) void compact_refs(Compact c) {
  const int64_t pairs = c.totals[0], live = *c.live;
  for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < c.n_pages; i += (int64_t)gridDim.x * kThreads) {
    if (c.refs_out != c.refs && (i < live) == (c.refs[i] != 0)) c.refs_out[i] = c.refs[i];
    if (i < pairs) {
      const int32_t from = c.from[i], to = c.to[i], refs = c.refs[from];
      c.refs_out[to] = refs;
      c.refs_out[from] = 0;
      c.places[from] = to;
    }
  }
}
// All of the books by one workgroup.
__global__ __launch_bounds__(kSoloThreads) void compact_solo(Compact c) {
  __shared__ int32_t from[kSoloPages / 2], to[kSoloPages / 2], refs_of[kSoloPages / 2], staying;
  __shared__ Pair shared[kSoloWaves];
  const int t = threadIdx.x, pages = c.n_pages, each = each_of(pages); // a lane's pages lie one after another
  i32x4 refs[kSoloEach / 4];
  Pair mine = {0, 0}, all;
#pragma unroll
  for (int k = 0; k < kSoloEach; k += 4)
    if (k < each) refs[k / 4] = four_of(c.refs, t * each + k, pages, 0);
#pragma unroll
  for (int k = 0; k < kSoloEach; ++k)
    if (k < each) mine.a += refs[k / 4][k % 4] != 0;
  int32_t before = sums_before(mine, shared, &all).a; // in use in front of a page
  const int32_t live = all.a;
  if (live >= t * each && live < (t + 1) * each) { // those in use below number `live`, which stay
    int32_t n = before;
#pragma unroll
    for (int k = 0; k < kSoloEach; ++k)
      if (k < each && t * each + k < live) n += refs[k / 4][k % 4] != 0;
    staying = n;
  }
  if (t == 0 && live >= kSoloThreads * each) staying = live;
  __syncthreads();
  const int32_t stay = staying;
#pragma unroll
  for (int k = 0; k < kSoloEach; ++k) {
    const int i = t * each + k;
    if (k >= each || i >= pages) continue;
    const int32_t n = refs[k / 4][k % 4];
    if (n && i >= live) from[before - stay] = i, refs_of[before - stay] = n;
    else if (!n && i < live) to[i - before] = i;
    else c.refs_out[i] = n;
    if (!(n && i >= live)) c.places[i] = n ? i : -1;
    before += n != 0;
  }
  __syncthreads();
  for (int k = t; k < live - stay; k += kSoloThreads) {
    const int32_t a = from[k], b = to[k];
    c.from[k] = a, c.to[k] = b;
    c.refs_out[b] = refs_of[k], c.refs_out[a] = 0;
    c.places[a] = b;
  }
  if (t == 0) c.totals[0] = live - stay, *c.live = live;
}
// entry_wgs: workgroups that rewrite tables; the others copy
template <int kVec> __global__ __launch_bounds__(kThreads) void compact_apply(Compact c, Buffers buffers, Shape shape, int32_t page_tokens, uint32_t entry_wgs, uint32_t parts) {
  if (blockIdx.x < entry_wgs) {
    for (int k = 0; k < HF_MAX_TABLES; ++k)
      for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < c.n_entries[k]; i += (int64_t)entry_wgs * kThreads) {
        const int32_t p = c.entries[k][i];
        c.entries_out[k][i] = p >= 0 && p < c.n_pages ? c.places[p] : p;
      }
    return;
  }
  each_part(c.totals[0], buffers.n, parts, blockIdx.x - entry_wgs, gridDim.x - entry_wgs, [&](int64_t k, uint32_t b, uint32_t part) {
    Part<kVec, true> data;
    data.load(buffers.at[b], shape, c.from[k], page_tokens, part);
    data.store(buffers.at[b], shape, c.to[k]);
  });
}

// ---- on the host ---------------------------------------------------------------------------------------------------------

int shift_of(int64_t n) { // n = 2^s
  int s = 0;
  while ((int64_t(1) << s) < n) ++s;
  return s;
}

Shape shape_of(const hf_kv_cache &c) {
  Shape s = {c.page_stride, 0, 0, 1, 1, c.head_dim, 1};
  const int64_t heads = c.n_kv_heads, dim = c.head_dim;
  if (c.token_stride == dim) { // a head's tokens in one run
    s.outer = (int32_t)heads, s.outer_stride = c.head_stride, s.growing = 2;
  } else if (c.head_stride == dim || heads == 1) { // a token's heads in one run
    s.inner = (int32_t)(heads * dim);
    if (c.token_stride == heads * dim) s.growing = 2;
    else s.growing = 0, s.outer_stride = c.token_stride;
  } else {
    s.outer = (int32_t)heads, s.outer_stride = c.head_stride, s.middle_stride = c.token_stride, s.growing = 1;
  }
  return s;
}
Buffers buffers_of(const hf_page_pool &pool) {
  Buffers b = {};
  for (int i = 0; i < pool.n_caches; ++i) b.at[b.n++] = pool.caches[i].k, b.at[b.n++] = pool.caches[i].v;
  return b;
}
// f(elements of an access, workgroups' shares of a whole page): 8 at a time where the shortest run has as many
template <typename F> hipError_t by_access(const Shape &s, int32_t page_tokens, const F &f) {
  const int vec = s.inner >= 8 ? 8 : 1;
  const int64_t runs = (int64_t)s.outer * s.middle * (s.growing < 2 ? page_tokens : 1), inner = s.growing == 2 ? (int64_t)s.inner * page_tokens : s.inner;
  const uint32_t parts = (uint32_t)up(runs * up(inner, vec), kThreads * kInFlight);
  return vec == 8 ? f(std::integral_constant<int, 8>{}, parts) : f(std::integral_constant<int, 1>{}, parts);
}
constexpr int64_t kMostRowWgs = 2048;
// Workgroups that copy: how much there is to do only the GPU knows, and those that find nothing cost time too.  us at 8192 / 10240 / 12288 / 16384, call after call from Python: rows that go on as they are, 256 of
// them over 80 layers 13.7 / 15.0 / 16.5 / 19.2, 64 over 32 layers 12.4 / 13.5 / 14.9 / 17.7, 1024 over 20 layers 21.4 / 22.8 / 24.2 / 27.2; the fork as above 73.8 / 73.6 / 73.0 / 71.0 (replayed from a graph
// 69.1 / 70.5 / 69.6 / 69.5).  Most steps of a rollout fork rows that go on as they are.  Where more rows come out than went in, some branch: 16 prompts into 64 samples each over 8 layers of 8 heads
// 339 / 335 / 334 / 331.  Compact as above at 4096 / 8192 / 16384 199 / 191 / 184, 1024 pages in use and none to move 6.6 / 8.5 / 11.7.
constexpr int64_t kMostCopyWgs = 16384, kMostForkWgs = 8192;
// One workgroup keeps the books of up to kSoloPages pages and kSoloEntries entries of tables (of tables and slots, twice as many): us, by one / by launches after one another, fork of 256 rows of 8, 31
// and 60 pages 8.8 / 16.1, 16.0 / 17.3, 25.5 / 17.8; grow by one token of 256 rows in 4096 and 16384 pages 8.0 / 10.2, 15.1 / 10.8, by 900 of 16 rows 10.5 / 12.6; compact of 1024, 8192 and 16384 pages
// 7.5 / 13.7, 16.3 / 18.7, 26.9 / 23.8.
constexpr int64_t kSoloEntries = 8192;

// arrays of a workspace, one after another, each 16-byte aligned
struct Room {
  uintptr_t at;
  size_t size = 0;
  template <typename T> T *take(int64_t n) {
    T *p = reinterpret_cast<T *>(at + size);
    size += up(n * sizeof(T), 16) * 16;
    return p;
  }
};
Tables tables_of(const hf_page_pool &pool, const int32_t *entries, const int32_t *lens, int32_t rows, int32_t width) {
  const hf_kv_cache &c = pool.caches[0];
  return {entries, lens, rows, width, shift_of(c.page_tokens), (int32_t)c.n_pages};
}
Fork fork_of(const hf_page_pool &pool, const hf_page_fork &a, Room &room) {
  Fork f = {tables_of(pool, a.tables, a.lens, a.rows, a.width), a.parents, a.refs, a.tables_out, a.lens_out, a.refs_out, a.rows_out};
  f.page_tile = tile_of(f.from.n_pages, kPageTile), f.row_tile = tile_of(a.rows_out, kRowTile);
  f.page_tiles = (int32_t)up(f.from.n_pages, f.page_tile), f.row_tiles = (int32_t)up(a.rows_out, f.row_tile);
  f.first = room.take<int32_t>(f.from.n_pages);
  f.free_sums = room.take<int64_t>(f.page_tiles);
  f.want_sums = room.take<int64_t>(f.row_tiles);
  f.free_list = room.take<int32_t>(a.rows_out);
  f.want = room.take<int32_t>(a.rows_out);
  f.moves = room.take<Move>(a.rows_out);
  f.totals = room.take<int64_t>(2);
  return f;
}
Grow grow_of(const hf_page_pool &pool, const hf_page_grow &a, Room &room) {
  Grow g = {tables_of(pool, a.tables, a.lens, a.rows, a.width), a.counts, a.refs, a.tables_out, a.lens_out, a.refs_out, a.slots, a.most};
  g.page_tile = tile_of(g.from.n_pages, kPageTile), g.row_tile = tile_of(a.rows, kRowTile);
  g.page_tiles = (int32_t)up(g.from.n_pages, g.page_tile), g.row_tiles = (int32_t)up(a.rows, g.row_tile);
  const int64_t each = std::min<int64_t>(a.width, up(a.most, int64_t(1) << g.from.shift)); // a row's fresh pages, at most
  g.list = std::min<int64_t>(g.from.n_pages, a.rows * each);
  g.free_sums = room.take<int64_t>(g.page_tiles);
  g.want_sums = room.take<int64_t>(g.row_tiles);
  g.before = room.take<int64_t>(a.rows);
  g.free_list = room.take<int32_t>(g.list);
  g.totals = room.take<int64_t>(1);
  return g;
}
Compact compact_of(const hf_page_pool &pool, const hf_page_compact &a, Room &room) {
  Compact c = {a.refs, a.refs_out, a.places, a.live};
  for (int k = 0; k < HF_MAX_TABLES; ++k) c.entries[k] = a.entries[k], c.entries_out[k] = a.entries_out[k], c.n_entries[k] = a.n_entries[k];
  c.n_pages = (int32_t)pool.caches[0].n_pages;
  c.page_tile = tile_of(c.n_pages, kPageTile), c.page_tiles = (int32_t)up(c.n_pages, c.page_tile);
  c.live_sums = room.take<int64_t>(c.page_tiles);
  c.from = room.take<int32_t>(c.n_pages / 2);
  c.to = room.take<int32_t>(c.n_pages / 2);
  c.totals = room.take<int64_t>(1);
  return c;
}

} // namespace

size_t fork_workspace(const hf_page_pool &pool, const hf_page_fork &a) {
  Room room = {0};
  fork_of(pool, a, room);
  return room.size;
}
size_t grow_workspace(const hf_page_pool &pool, const hf_page_grow &a) {
  Room room = {0};
  grow_of(pool, a, room);
  return room.size;
}
size_t compact_workspace(const hf_page_pool &pool, const hf_page_compact &a) {
  Room room = {0};
  compact_of(pool, a, room);
  return room.size;
}

int launch_fork(const hf_page_pool &pool, const hf_page_fork &a, void *stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  Room room = {reinterpret_cast<uintptr_t>(a.workspace)};
  const Fork f = fork_of(pool, a, room);
  const auto wgs = [](int64_t n, int64_t each) { return dim3((uint32_t)std::max<int64_t>(1, std::min(up(n, each), kMostRowWgs))); };
  const bool solo = f.from.n_pages <= kSoloPages && std::max(a.rows, a.rows_out) <= kSoloRows && (int64_t)std::max(a.rows, a.rows_out) * a.width <= kSoloEntries;
  if (solo) {
    if (const hipError_t e = enqueue_kernel(fork_solo, dim3(1), kSoloThreads, st, f)) return e;
  } else {
    if (const hipError_t e = enqueue_kernel(fork_begin, wgs(f.from.n_pages, kThreads), kThreads, st, f)) return e;
    if (const hipError_t e = enqueue_kernel(fork_count, wgs((int64_t)a.rows + a.rows_out, kWaves), kThreads, st, f)) return e;
    if (const hipError_t e = enqueue_kernel(fork_sums, dim3(f.page_tiles + f.row_tiles), kThreads, st, f)) return e;
    if (const hipError_t e = enqueue_kernel(fork_lists, dim3(f.page_tiles + f.row_tiles), kThreads, st, f)) return e;
  }
  const uint32_t row_wgs = solo ? 0 : wgs(a.rows_out, kWaves).x;
  const Shape shape = shape_of(pool.caches[0]);
  return by_access(shape, pool.caches[0].page_tokens, [&](auto vec, uint32_t parts) {
    const int64_t copies = std::min((int64_t)a.rows_out * 2 * pool.n_caches * parts, a.rows_out > a.rows ? kMostCopyWgs : kMostForkWgs);
    if (row_wgs + copies == 0) return hipSuccess;
    return enqueue_kernel(fork_apply<decltype(vec)::value>, dim3(row_wgs + (uint32_t)copies), kThreads, st, f, buffers_of(pool), shape, row_wgs, parts);
  });
}

int launch_grow(const hf_page_pool &pool, const hf_page_grow &a, void *stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  Room room = {reinterpret_cast<uintptr_t>(a.workspace)};
  const Grow g = grow_of(pool, a, room);
  if (g.from.n_pages <= kSoloPages && a.rows <= kSoloRows && g.list <= kSoloFresh && (int64_t)a.rows * ((int64_t)a.width + a.most) <= 2 * kSoloEntries)
    return enqueue_kernel(grow_solo, dim3(1), kSoloThreads, st, g);
  if (const hipError_t e = enqueue_kernel(grow_sums, dim3(g.page_tiles + g.row_tiles), kThreads, st, g)) return e;
  if (const hipError_t e = enqueue_kernel(grow_lists, dim3(g.page_tiles + g.row_tiles), kThreads, st, g)) return e;
  return enqueue_kernel(grow_apply, dim3((uint32_t)std::max<int64_t>(1, std::min(up(a.rows, kWaves), kMostRowWgs))), kThreads, st, g);
}

int launch_compact(const hf_page_pool &pool, const hf_page_compact &a, void *stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  Room room = {reinterpret_cast<uintptr_t>(a.workspace)};
  const Compact c = compact_of(pool, a, room);
  if (c.n_pages <= kSoloPages) {
    if (const hipError_t e = enqueue_kernel(compact_solo, dim3(1), kSoloThreads, st, c)) return e;
  } else {
    if (const hipError_t e = enqueue_kernel(compact_sums, dim3(c.page_tiles), kThreads, st, c)) return e;
    if (const hipError_t e = enqueue_kernel(compact_lists, dim3(c.page_tiles), kThreads, st, c)) return e;
    if (const hipError_t e = enqueue_kernel(compact_refs, dim3((uint32_t)std::min(up(c.n_pages, kThreads), kMostRowWgs)), kThreads, st, c)) return e;
  }
  int64_t most = 0;
  for (const int64_t n : c.n_entries) most = std::max(most, n);
  const uint32_t entry_wgs = (uint32_t)std::min(up(most, kThreads), kMostRowWgs);
  const Shape shape = shape_of(pool.caches[0]);
  return by_access(shape, pool.caches[0].page_tokens, [&](auto vec, uint32_t parts) {
    const int64_t copies = std::min((int64_t)c.n_pages / 2 * 2 * pool.n_caches * parts, kMostCopyWgs);
    if (entry_wgs + copies == 0) return hipSuccess;
    return enqueue_kernel(compact_apply<decltype(vec)::value>, dim3(entry_wgs + (uint32_t)copies), kThreads, st, c, buffers_of(pool), shape, pool.caches[0].page_tokens, entry_wgs, parts);
  });
}

} // namespace hf
