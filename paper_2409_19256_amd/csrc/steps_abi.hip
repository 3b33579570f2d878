// C entry points of what surrounds a rollout's steps (declarations and contracts: include/hfreshard.h): the checks of what they are given.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "checks.hpp"
#include "step_kernels.hpp"

// the Python binding mirrors these layouts field by field
static_assert(sizeof(hf_adjustment) == 160 && sizeof(hf_distillation) == 56 && sizeof(hf_distillation_grad) == 56, "ABI struct layout");
static_assert(sizeof(hf_page_pool) == 16 && sizeof(hf_page_fork) == 88 && sizeof(hf_page_grow) == 96 && sizeof(hf_page_compact) == 144, "ABI struct layout");

namespace {

using hf::set_error;
using namespace hf::check;

int64_t size_of(int dtype) { return dtype == HF_F32 ? 4 : 2; }

int check_adjustment(const hf_adjustment *p) {
  if (!p) return set_error(HF_EINVAL, "null arguments");
  const hf_adjustment &a = *p;
  if (a.dtype != HF_BF16 && a.dtype != HF_F16 && a.dtype != HF_F32) return set_error(HF_EINVAL, "unknown type of logits");
  if (a.rows < 0 || a.width < 0 || a.n_bias < 0 || a.n_allowed < 0) return set_error(HF_EINVAL, "negative size");
  if (a.vocab < 1 || a.vocab > (1 << 30)) return set_error(HF_EINVAL, "vocab must be in [1, 2^30]");
  if (a.rows == 0) return HF_OK;
  if (!a.logits || !a.out) return set_error(HF_EINVAL, "null logits or output");
  if (!a.tokens != !a.lens) return set_error(HF_EINVAL, "tokens and lens go together");
  if (a.tokens && a.token_bytes != 4 && a.token_bytes != 8) return set_error(HF_EINVAL, "token_bytes must be 4 or 8");
  if (a.n_bias && (!a.bias_ids || !a.bias)) return set_error(HF_EINVAL, "biases need their ids and values");
  const size_t size = size_of(a.dtype);
  if (!aligned(a.logits, size) || !aligned(a.out, size) || (a.tokens && !aligned(a.tokens, a.token_bytes)) || !aligned(a.lens, 4) || !aligned(a.prompt_lens, 4) ||
      !aligned(a.repetition, 4) || !aligned(a.frequency, 4) || !aligned(a.presence, 4) || !aligned(a.bias_ids, 4) || !aligned(a.bias, 4) || !aligned(a.allowed, 4) ||
      !aligned(a.allowed_rows, 4))
    return set_error(HF_EINVAL, "arrays must be aligned to their elements");
  const int64_t words = (a.vocab + 31) / 32;
  const Dim from[] = {{a.rows, a.row_stride}}, to[] = {{a.rows, a.out_stride}}, tokens[] = {{a.rows, a.tokens_stride}}, allowed[] = {{a.n_allowed, a.allowed_stride}};
  if (!span(from, a.vocab) || !span(to, a.vocab)) return set_error(HF_EINVAL, "row_stride or out_stride is negative or spans too much");
  if (a.tokens && a.width && !span(tokens, a.width)) return set_error(HF_EINVAL, "tokens_stride is negative or spans too much");
  if (a.allowed && !span(allowed, words)) return set_error(HF_EINVAL, "allowed_stride is negative or spans too much");
  if (!separate(to, a.vocab)) return set_error(HF_EINVAL, "the output overlaps itself");
  if (a.width > hf::kMaxAdjustList || a.n_bias > hf::kMaxAdjustList) return set_error(HF_ERANGE, "width and n_bias must be at most 2^31 - 512");
  if (!hf::adjust_fits(a)) return set_error(HF_ERANGE, "too many rows for one launch");
  const bool same = a.logits == a.out && (a.rows == 1 || a.row_stride == a.out_stride);
  const int64_t biases = a.n_bias > INT64_MAX / a.rows ? INT64_MAX : a.rows * a.n_bias;
  const Output outputs[] = {{"the output overlaps an input and is not the logits", place(a.out, to, a.vocab, size)}};
  if (const char *what = first_overlap(outputs, {same ? Place{} : place(a.logits, from, a.vocab, size),
                                                 a.tokens && a.width ? place(a.tokens, tokens, a.width, a.token_bytes) : Place{}, array(a.lens, a.rows, 4),
                                                 array(a.prompt_lens, a.rows, 4), array(a.repetition, a.rows, 4), array(a.frequency, a.rows, 4),
                                                 array(a.presence, a.rows, 4), array(a.bias_ids, biases, 4), array(a.bias, biases, 4),
                                                 a.allowed ? place(a.allowed, allowed, words, 4) : Place{}, array(a.allowed_rows, a.allowed ? a.rows : 0, 4)}))
    return set_error(HF_EINVAL, what);
  return HF_OK;
}

// The caches of a pool, all alike.
int check_pool(const hf_page_pool *p) {
  if (!p || !p->caches) return set_error(HF_EINVAL, "null pool");
  if (p->n_caches < 1 || p->n_caches > HF_MAX_CACHES) return set_error(HF_EINVAL, "n_caches must be in [1, HF_MAX_CACHES]");
  const hf_kv_cache &c = p->caches[0];
  if (int rc = check_cache(&c)) return rc;
  for (int i = 1; i < p->n_caches; ++i) {
    const hf_kv_cache &d = p->caches[i];
    if (!d.k || !d.v || !aligned(d.k, 2) || !aligned(d.v, 2)) return set_error(HF_EINVAL, "null or misaligned cache buffer");
    if (d.dtype != c.dtype || d.n_kv_heads != c.n_kv_heads || d.head_dim != c.head_dim || d.page_tokens != c.page_tokens || d.n_pages != c.n_pages ||
        d.page_stride != c.page_stride || d.head_stride != c.head_stride || d.token_stride != c.token_stride)
      return set_error(HF_EINVAL, "the caches of a pool have to be alike");
  }
  return HF_OK;
}

// The first cache's keys, as a place in memory.
Place first_of(const hf_page_pool &pool) {
  const hf_kv_cache &c = pool.caches[0];
  const Dim dims[] = {{c.n_pages, c.page_stride}, {c.n_kv_heads, c.head_stride}, {c.page_tokens, c.token_stride}};
  Place p = place(c.k, dims, c.head_dim, 2);
  for (const int i : {2, 1, 2}) // what of a page lies in one run is one run, so that an array of several tokens' size still has an exact answer
    if (p.dims[i].n > 1 && p.dims[i].stride == p.inner) p.inner *= p.dims[i].n, p.dims[i] = {1, 0};
  return p;
}

// Keys and values of a pool's caches, as places in memory: all alike but for where they begin.
class Buffers {
  Place one_;
  uintptr_t begins_[2 * HF_MAX_CACHES]; // ascending
  int n_ = 0;
  bool apart_ = true; // one ends before the next begins
  Place at(uintptr_t begin) const {
    Place p = one_;
    p.end += begin - p.begin, p.begin = begin;
    return p;
  }
  void sort() {
    if (!std::is_sorted(begins_, begins_ + n_)) std::sort(begins_, begins_ + n_);
  }

public:
  explicit Buffers(const hf_page_pool &pool) {
    one_ = first_of(pool);
    for (int i = 0; i < pool.n_caches; ++i)
      for (const void *p : {pool.caches[i].k, pool.caches[i].v}) begins_[n_++] = reinterpret_cast<uintptr_t>(p);
    sort();
    for (int i = 1; i < n_; ++i) apart_ = apart_ && begins_[i] - begins_[i - 1] >= one_.end - one_.begin;
  }
  bool meet(const Place &p) const {
    const uintptr_t *end = std::lower_bound(begins_, begins_ + n_, p.end), *b = begins_; // those that begin before it ends
    if (apart_) b = std::lower_bound(b, end, p.begin - std::min(p.begin, one_.end - one_.begin));
    return std::any_of(b, end, [&](uintptr_t q) { return overlap(p, at(q)); });
  }
  // Whether two of them share a byte.  Mostly they lie one after another; where they lie between one another's pages, only those whose beginnings are
  // nearer than a page's own span, page strides left out, have to be looked at.
  bool meet_one_another() {
    if (apart_) return false;
    const Dim &pages = one_.dims[0], &heads = one_.dims[1], &tokens = one_.dims[2];
    const int64_t reach = (heads.n - 1) * heads.stride + (tokens.n - 1) * tokens.stride + one_.inner;
    const uintptr_t period = pages.n > 1 && pages.stride >= reach ? pages.stride : 0;
    struct Begin {
      uintptr_t in_period, at;
    } begins[2 * HF_MAX_CACHES];
    for (int i = 0; i < n_; ++i) begins[i] = {period ? begins_[i] % period : begins_[i], begins_[i]};
    std::sort(begins, begins + n_, [](const Begin &x, const Begin &y) { return x.in_period < y.in_period; });
    for (int i = 0; i < n_; ++i)
      for (int k = 1; k < n_; ++k) {
        const int j = (i + k) % n_;
        if (!period && j < i) break;
        if (period && begins[j].in_period + (j < i ? period : 0) - begins[i].in_period >= (uint64_t)reach) break;
        if (overlap(at(begins[i].at), at(begins[j].at))) return true;
      }
    return false;
  }
};

// Whether an output of a call that leaves the caches alone lies in one of them.  Mostly all outputs are near one another and no cache is: one look at every buffer.
template <size_t kN> bool in_a_cache(const hf_page_pool &pool, const Output (&outputs)[kN]) {
  Place one = first_of(pool);
  const uintptr_t size = one.end - one.begin;
  uintptr_t begin = UINTPTR_MAX, end = 0;
  for (const Output &o : outputs)
    if (o.place.end) begin = std::min(begin, o.place.begin), end = std::max(end, o.place.end);
  for (int i = 0; i < pool.n_caches; ++i)
    for (const void *p : {pool.caches[i].k, pool.caches[i].v}) {
      one.begin = reinterpret_cast<uintptr_t>(p), one.end = one.begin + size;
      if (one.begin >= end || begin >= one.end) continue;
      for (const Output &o : outputs)
        if (overlap(one, o.place)) return true;
    }
  return false;
}

// a page in one buffer has to be countable in 32 bits
int check_moves(const hf_page_pool &pool) {
  const hf_kv_cache &c = pool.caches[0];
  if ((unsigned __int128)c.n_kv_heads * c.page_tokens * c.head_dim > INT32_MAX) return set_error(HF_ERANGE, "a page is too large");
  return HF_OK;
}

int64_t of_rows(int64_t rows, int64_t width) { return width && rows > INT64_MAX / width ? INT64_MAX : rows * width; }

int check_workspace(const void *workspace, size_t bytes, size_t need) {
  if (!workspace || !aligned(workspace, 16)) return set_error(HF_EINVAL, "the workspace must be given and 16-byte aligned");
  if (bytes < need) return set_error(HF_EINVAL, "the workspace is smaller than its ..._workspace_bytes says");
  return HF_OK;
}

int check_fork(const hf_page_pool *pool, const hf_page_fork *a) {
  if (int rc = check_pool(pool)) return rc;
  if (!a) return set_error(HF_EINVAL, "null arguments");
  if (a->rows < 0 || a->rows_out < 0 || a->width < 0) return set_error(HF_EINVAL, "negative size");
  if ((int64_t)a->rows + a->rows_out > INT32_MAX / 2) return set_error(HF_ERANGE, "too many rows");
  return check_moves(*pool);
}
int check_grow(const hf_page_pool *pool, const hf_page_grow *a) {
  if (int rc = check_pool(pool)) return rc;
  if (!a) return set_error(HF_EINVAL, "null arguments");
  if (a->rows < 0 || a->width < 0 || a->most < 0) return set_error(HF_EINVAL, "negative size");
  if (a->rows > INT32_MAX / 2) return set_error(HF_ERANGE, "too many rows");
  return HF_OK;
}
int check_compact(const hf_page_pool *pool, const hf_page_compact *a) {
  if (int rc = check_pool(pool)) return rc;
  if (!a) return set_error(HF_EINVAL, "null arguments");
  for (const int64_t n : a->n_entries)
    if (n < 0 || n > (int64_t)1 << 40) return set_error(HF_EINVAL, "a number of entries is negative or too large");
  return check_moves(*pool);
}

} // namespace

extern "C" {

int hf_adjust_logits(const hf_adjustment *args, void *hip_stream) {
  if (int rc = check_adjustment(args)) return rc;
  if (args->rows == 0) return HF_OK;
  return launched(hf::launch_adjust(*args, hip_stream));
}

int hf_top_distill(const hf_logits *in, const hf_distillation *args, void *hip_stream) {
  if (int rc = check_logits(in)) return rc;
  if (!args) return set_error(HF_EINVAL, "null arguments");
  const hf_distillation &a = *args;
  if (in->targets) return set_error(HF_EINVAL, "targets have no part in this");
  if (a.n < 1 || a.n > HF_MAX_DISTILL) return set_error(HF_EINVAL, "n must be in [1, HF_MAX_DISTILL]");
  if (!(a.reverse >= 0 && a.reverse <= 1)) return set_error(HF_EINVAL, "reverse must be in [0, 1]");
  if (a.flags & ~HF_DISTILL_REST) return set_error(HF_EINVAL, "unknown flag");
  if (!a.norm != !a.slopes) return set_error(HF_EINVAL, "norm and slopes go together");
  if (in->rows == 0) return HF_OK;
  if (!a.ids || !a.logprobs) return set_error(HF_EINVAL, "null ids or log probabilities");
  if (!aligned(a.ids, 4) || !aligned(a.logprobs, 4) || !aligned(a.loss, 4) || !aligned(a.norm, 4) || !aligned(a.slopes, 4))
    return set_error(HF_EINVAL, "arrays must be aligned to their elements");
  if ((uint64_t)in->rows > hf::kMaxWgs / 4) return set_error(HF_ERANGE, "too many rows for one launch"); // workgroups of up to 1024 lanes
  const Dim from[] = {{in->rows, in->row_stride}};
  const Output outputs[] = {{"loss overlaps an input", array(a.loss, in->rows, 4)},
                            {"norm overlaps an input or another output", array(a.norm, 2 * in->rows, 4)},
                            {"slopes overlap an input or another output", array(a.slopes, in->rows * (a.n + 1), 4)}};
  if (const char *what = first_overlap(outputs, {place(in->logits, from, in->vocab, size_of(in->dtype)), array(a.ids, in->rows * a.n, 4), array(a.logprobs, in->rows * a.n, 4)}))
    return set_error(HF_EINVAL, what);
  return launched(hf::launch_top_distill(*in, a, hip_stream));
}

int hf_top_distill_back(const hf_logits *in, const hf_distillation_grad *grad, void *hip_stream) {
  if (int rc = check_logits(in)) return rc;
  if (!grad) return set_error(HF_EINVAL, "null arguments");
  const hf_distillation_grad &g = *grad;
  if (in->targets) return set_error(HF_EINVAL, "targets have no part in this");
  if (g.n < 1 || g.n > HF_MAX_DISTILL) return set_error(HF_EINVAL, "n must be in [1, HF_MAX_DISTILL]");
  if (in->rows == 0) return HF_OK;
  const size_t size = size_of(in->dtype);
  if (!g.ids || !g.norm || !g.slopes || !g.grad_loss || !g.dlogits) return set_error(HF_EINVAL, "null ids, norm, slopes, grad_loss or dlogits");
  if (!aligned(g.ids, 4) || !aligned(g.norm, 4) || !aligned(g.slopes, 4) || !aligned(g.grad_loss, 4) || !aligned(g.dlogits, size))
    return set_error(HF_EINVAL, "arrays must be aligned to their elements");
  const Dim from[] = {{in->rows, in->row_stride}}, to[] = {{in->rows, g.dlogits_stride}};
  if (!span(to, in->vocab)) return set_error(HF_EINVAL, "dlogits_stride is negative or spans too much");
  if (!separate(to, in->vocab)) return set_error(HF_EINVAL, "dlogits overlaps itself");
  if ((uint64_t)in->rows > hf::kMaxWgs || (uint64_t)in->rows * hf::distill_back_segments(*in) > hf::kMaxWgs)
    return set_error(HF_ERANGE, "too many rows for one launch");
  const bool same = in->logits == g.dlogits && (in->rows == 1 || in->row_stride == g.dlogits_stride);
  const Output outputs[] = {{"dlogits overlaps an input and is not the logits", place(g.dlogits, to, in->vocab, size)}};
  if (const char *what = first_overlap(outputs, {same ? Place{} : place(in->logits, from, in->vocab, size), array(g.ids, in->rows * g.n, 4), array(g.norm, 2 * in->rows, 4),
                                                 array(g.slopes, in->rows * (g.n + 1), 4), array(g.grad_loss, in->rows, 4)}))
    return set_error(HF_EINVAL, what);
  return launched(hf::launch_top_distill_back(*in, g, hip_stream));
}

size_t hf_fork_pages_workspace_bytes(const hf_page_pool *pool, const hf_page_fork *args) {
  if (check_fork(pool, args)) return (size_t)-1;
  return hf::fork_workspace(*pool, *args);
}

int hf_fork_pages(const hf_page_pool *pool, const hf_page_fork *args, void *hip_stream) {
  if (int rc = check_fork(pool, args)) return rc;
  const hf_page_fork &a = *args;
  const bool old = a.rows > 0, out = a.rows_out > 0, wide = a.width > 0;
  if ((old && (!a.lens || (wide && !a.tables))) || (out && (!a.parents || !a.lens_out || (wide && !a.tables_out))) || !a.refs || !a.refs_out)
    return set_error(HF_EINVAL, "null tables, lengths, parents or reference counts");
  if (!aligned(a.tables, 4) || !aligned(a.lens, 4) || !aligned(a.parents, 4) || !aligned(a.refs, 4) || !aligned(a.tables_out, 4) || !aligned(a.lens_out, 4) ||
      !aligned(a.refs_out, 4))
    return set_error(HF_EINVAL, "arrays must be aligned to their elements");
  const size_t need = hf::fork_workspace(*pool, a);
  const int64_t pages = pool->caches[0].n_pages;
  const Place tables = array(old ? a.tables : nullptr, of_rows(a.rows, a.width), 4), lens = array(a.lens, a.rows, 4), parents = array(a.parents, a.rows_out, 4),
              refs = array(a.refs, pages, 4);
  const Output outputs[] = {{"tables_out overlaps an input", array(out ? a.tables_out : nullptr, of_rows(a.rows_out, a.width), 4)},
                            {"lens_out overlaps an input or another output", array(a.lens_out, a.rows_out, 4)},
                            {"the workspace overlaps an input or an output", array(a.workspace, (int64_t)need, 1)},
                            {"refs_out overlaps an input or another output and is not refs", array(a.refs_out, pages, 4)}};
  if (const char *what = first_overlap(outputs, {tables, lens, parents, a.refs == a.refs_out ? Place{} : refs})) return set_error(HF_EINVAL, what);
  Buffers buffers(*pool);
  for (const Place &p : {tables, lens, parents, refs})
    if (buffers.meet(p)) return set_error(HF_EINVAL, "a cache overlaps an input");
  for (const Output &o : outputs)
    if (buffers.meet(o.place)) return set_error(HF_EINVAL, "a cache overlaps an output");
  if (buffers.meet_one_another()) return set_error(HF_EINVAL, "the caches overlap one another");
  if (int rc = check_workspace(a.workspace, a.workspace_bytes, need)) return rc;
  return launched(hf::launch_fork(*pool, a, hip_stream));
}

size_t hf_grow_pages_workspace_bytes(const hf_page_pool *pool, const hf_page_grow *args) {
  if (check_grow(pool, args)) return (size_t)-1;
  return hf::grow_workspace(*pool, *args);
}

int hf_grow_pages(const hf_page_pool *pool, const hf_page_grow *args, void *hip_stream) {
  if (int rc = check_grow(pool, args)) return rc;
  const hf_page_grow &a = *args;
  const bool rows = a.rows > 0, wide = a.width > 0;
  if ((rows && (!a.lens || !a.counts || !a.lens_out || (wide && (!a.tables || !a.tables_out)) || (a.most && !a.slots))) || !a.refs || !a.refs_out)
    return set_error(HF_EINVAL, "null tables, lengths, counts, slots or reference counts");
  if (!aligned(a.tables, 4) || !aligned(a.lens, 4) || !aligned(a.counts, 4) || !aligned(a.refs, 4) || !aligned(a.tables_out, 4) || !aligned(a.lens_out, 4) ||
      !aligned(a.slots, 8) || !aligned(a.refs_out, 4))
    return set_error(HF_EINVAL, "arrays must be aligned to their elements");
  const size_t need = hf::grow_workspace(*pool, a);
  const int64_t pages = pool->caches[0].n_pages;
  const Place tables = array(rows ? a.tables : nullptr, of_rows(a.rows, a.width), 4), lens = array(a.lens, a.rows, 4), counts = array(a.counts, a.rows, 4),
              refs = array(a.refs, pages, 4);
  Output outputs[] = {{"tables_out overlaps an input and is not tables", array(rows ? a.tables_out : nullptr, of_rows(a.rows, a.width), 4)},
                      {"lens_out overlaps an input or another output and is not lens", array(a.lens_out, a.rows, 4)},
                      {"slots overlap an input or another output", array(rows ? a.slots : nullptr, of_rows(a.rows, a.most), 8)},
                      {"the workspace overlaps an input or an output", array(a.workspace, (int64_t)need, 1)},
                      {"refs_out overlaps an input or another output and is not refs", array(a.refs_out, pages, 4)}};
  // what is written where it was read meets no other output either
  if (const char *what = first_overlap(outputs, {a.tables == a.tables_out ? Place{} : tables, a.lens == a.lens_out ? Place{} : lens, counts, a.refs == a.refs_out ? Place{} : refs}))
    return set_error(HF_EINVAL, what);
  if (in_a_cache(*pool, outputs)) return set_error(HF_EINVAL, "a cache overlaps an output");
  if (int rc = check_workspace(a.workspace, a.workspace_bytes, need)) return rc;
  return launched(hf::launch_grow(*pool, a, hip_stream));
}

size_t hf_compact_pages_workspace_bytes(const hf_page_pool *pool, const hf_page_compact *args) {
  if (check_compact(pool, args)) return (size_t)-1;
  return hf::compact_workspace(*pool, *args);
}

int hf_compact_pages(const hf_page_pool *pool, const hf_page_compact *args, void *hip_stream) {
  if (int rc = check_compact(pool, args)) return rc;
  const hf_page_compact &a = *args;
  if (!a.refs || !a.refs_out || !a.places || !a.live) return set_error(HF_EINVAL, "null reference counts, places or live");
  if (!aligned(a.refs, 4) || !aligned(a.refs_out, 4) || !aligned(a.places, 4) || !aligned(a.live, 4)) return set_error(HF_EINVAL, "arrays must be aligned to their elements");
  for (int k = 0; k < HF_MAX_TABLES; ++k)
    if (a.n_entries[k] && (!a.entries[k] || !a.entries_out[k] || !aligned(a.entries[k], 4) || !aligned(a.entries_out[k], 4)))
      return set_error(HF_EINVAL, "null or misaligned entries");
  const size_t need = hf::compact_workspace(*pool, a);
  const int64_t pages = pool->caches[0].n_pages;
  const Place refs = array(a.refs, pages, 4);
  Place in[HF_MAX_TABLES], to[HF_MAX_TABLES];
  for (int k = 0; k < HF_MAX_TABLES; ++k) in[k] = array(a.entries[k], a.n_entries[k], 4), to[k] = array(a.entries_out[k], a.n_entries[k], 4);
  static_assert(HF_MAX_TABLES == 4, "all of them are named below");
  const Output outputs[] = {{"entries_out overlap another output", to[0]},
                            {"entries_out overlap another output", to[1]},
                            {"entries_out overlap another output", to[2]},
                            {"entries_out overlap another output", to[3]},
                            {"places overlap an input or another output", array(a.places, pages, 4)},
                            {"live overlaps an input or another output", array(a.live, 1, 4)},
                            {"the workspace overlaps an input or an output", array(a.workspace, (int64_t)need, 1)},
                            {"refs_out overlaps an input or another output and is not refs", array(a.refs_out, pages, 4)}};
  if (const char *what = first_overlap(outputs, {a.refs == a.refs_out ? Place{} : refs})) return set_error(HF_EINVAL, what);
  for (int i = 0; i < HF_MAX_TABLES; ++i)
    for (size_t j = 0; j < sizeof(outputs) / sizeof(outputs[0]); ++j)
      if (!((int)j == i && a.entries[i] == a.entries_out[i]) && overlap(in[i], outputs[j].place)) return set_error(HF_EINVAL, "entries overlap an output that is not their own");
  Buffers buffers(*pool);
  for (const Place &p : {refs, in[0], in[1], in[2], in[3]})
    if (buffers.meet(p)) return set_error(HF_EINVAL, "a cache overlaps an input");
  for (const Output &o : outputs)
    if (buffers.meet(o.place)) return set_error(HF_EINVAL, "a cache overlaps an output");
  if (buffers.meet_one_another()) return set_error(HF_EINVAL, "the caches overlap one another");
  if (int rc = check_workspace(a.workspace, a.workspace_bytes, need)) return rc;
  return launched(hf::launch_compact(*pool, a, hip_stream));
}

} // extern "C"
