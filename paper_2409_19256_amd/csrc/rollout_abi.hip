// C entry points of the rollout operators (declarations and contracts: include/hfreshard.h): the checks of what they are given.
#include <hip/hip_runtime.h>

#include <cmath>

#include "hfreshard.h"
#include "kernels.hpp"
#include "rollout_kernels.hpp"

// the Python binding mirrors these layouts field by field
static_assert(sizeof(hf_kv_cache) == 64 && sizeof(hf_append) == 152 && sizeof(hf_attention) == 152, "ABI struct layout");
static_assert(sizeof(hf_logits) == 48 && sizeof(hf_logprobs) == 56 && sizeof(hf_logprobs_grad) == 48, "ABI struct layout");

namespace {

using hf::set_error;

constexpr unsigned __int128 kMost = (unsigned __int128)1 << 60; // elements that a tensor may span

struct Dim {
  int64_t n, stride;
};

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// elements from the first to past the last of a tensor whose innermost `inner` are contiguous; 0 = a negative stride or a span beyond kMost
template <size_t kN> int64_t span(const Dim (&dims)[kN], int64_t inner) {
  unsigned __int128 all = inner;
  for (const Dim &d : dims) {
    if (d.n == 0) continue;
    if (d.stride < 0) return 0;
    all += (unsigned __int128)(d.n - 1) * (uint64_t)d.stride;
    if (all > kMost) return 0;
  }
  return (int64_t)all;
}

// whether no two elements of it share a place (the dimensions nest in some order)
template <size_t kN> bool separate(const Dim (&dims)[kN], int64_t inner) {
  unsigned __int128 need = inner;
  bool used[kN] = {};
  for (size_t k = 0; k < kN; ++k) { // by ascending stride
    size_t best = kN;
    for (size_t i = 0; i < kN; ++i)
      if (!used[i] && (best == kN || dims[i].stride < dims[best].stride)) best = i;
    used[best] = true;
    if (dims[best].n <= 1) continue;
    if ((unsigned __int128)dims[best].stride < need) return false;
    need += (unsigned __int128)(dims[best].n - 1) * (uint64_t)dims[best].stride;
  }
  return true;
}

bool overlap(const void *a, int64_t a_bytes, const void *b, int64_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + (uint64_t)b_bytes && y < x + (uint64_t)a_bytes;
}

// whether a tensor's vectors of `vec` 2-byte elements are aligned wherever they begin
template <size_t kN> bool divides(const void *p, const Dim (&dims)[kN], int vec) {
  if (!aligned(p, 2 * vec)) return false;
  for (const Dim &d : dims)
    if (d.n > 1 && d.stride % vec) return false;
  return true;
}

int check_cache(const hf_kv_cache *c) {
  if (!c) return set_error(HF_EINVAL, "null cache");
  if (!c->k || !c->v) return set_error(HF_EINVAL, "null cache buffer");
  if (c->k == c->v) return set_error(HF_EINVAL, "keys and values lie in the same place");
  if (c->dtype != HF_BF16 && c->dtype != HF_F16) return set_error(HF_EINVAL, "a cache is HF_BF16 or HF_F16");
  if (!aligned(c->k, 2) || !aligned(c->v, 2)) return set_error(HF_EINVAL, "cache buffers must be aligned to their elements");
  if (c->n_kv_heads < 1) return set_error(HF_EINVAL, "n_kv_heads must be positive");
  if (c->head_dim < 1 || c->head_dim > 256) return set_error(HF_EINVAL, "head_dim must be in [1, 256]");
  if (c->page_tokens < 4 || c->page_tokens > 65536 || (c->page_tokens & (c->page_tokens - 1)))
    return set_error(HF_EINVAL, "page_tokens must be a power of two in [4, 65536]");
  if (c->n_pages < 1 || c->n_pages > INT32_MAX) return set_error(HF_EINVAL, "n_pages must be in [1, 2^31 - 1]");
  const Dim dims[] = {{c->n_pages, c->page_stride}, {c->n_kv_heads, c->head_stride}, {c->page_tokens, c->token_stride}};
  if (!span(dims, c->head_dim)) return set_error(HF_EINVAL, "cache strides are negative or span too much");
  if (!separate(dims, c->head_dim)) return set_error(HF_EINVAL, "cache strides put two tokens in one place");
  return HF_OK;
}

int check_attention(const hf_kv_cache *c, const hf_attention *a) {
  if (int rc = check_cache(c)) return rc;
  if (!a) return set_error(HF_EINVAL, "null arguments");
  if (a->n_seqs < 0 || a->n_groups < 0 || a->max_group < 0 || a->prefix_width < 0 || a->suffix_width < 0 || a->max_prefix < 0 || a->max_suffix < 0)
    return set_error(HF_EINVAL, "negative size");
  if (a->n_q_heads < 1 || a->n_q_heads % c->n_kv_heads) return set_error(HF_EINVAL, "n_q_heads must be a multiple of n_kv_heads");
  if (!std::isfinite(a->scale)) return set_error(HF_EINVAL, "scale must be finite");
  if ((int64_t)a->n_seqs * a->n_q_heads > INT32_MAX / 2) return set_error(HF_ERANGE, "too many queries");
  return HF_OK;
}

int check_logits(const hf_logits *in) {
  if (!in) return set_error(HF_EINVAL, "null arguments");
  if (in->dtype != HF_BF16 && in->dtype != HF_F16 && in->dtype != HF_F32) return set_error(HF_EINVAL, "unknown type of logits");
  if (in->rows < 0) return set_error(HF_EINVAL, "negative size");
  if (in->vocab < 1 || in->vocab > (1 << 30)) return set_error(HF_EINVAL, "vocab must be in [1, 2^30]");
  if (!(in->inv_temperature > 0) || !std::isfinite(in->inv_temperature)) return set_error(HF_EINVAL, "inv_temperature must be positive and finite");
  if (in->rows == 0) return HF_OK;
  if (!in->logits) return set_error(HF_EINVAL, "null logits");
  const Dim dims[] = {{in->rows, in->row_stride}};
  if (!span(dims, in->vocab)) return set_error(HF_EINVAL, "row_stride is negative or spans too much");
  if (!aligned(in->logits, in->dtype == HF_F32 ? 4 : 2)) return set_error(HF_EINVAL, "logits must be aligned to their elements");
  if (in->targets && in->target_bytes != 4 && in->target_bytes != 8) return set_error(HF_EINVAL, "target_bytes must be 4 or 8");
  if (in->targets && !aligned(in->targets, in->target_bytes)) return set_error(HF_EINVAL, "targets must be aligned to their elements");
  return HF_OK;
}

int launched(int e) {
  if (e != 0) return set_error(HF_EHIP, hipGetErrorString(static_cast<hipError_t>(e)));
  return HF_OK;
}

bool attention_vec(const hf_kv_cache &c, const hf_attention &a) {
  const Dim cache[] = {{c.n_pages, c.page_stride}, {c.n_kv_heads, c.head_stride}, {c.page_tokens, c.token_stride}};
  const Dim q[] = {{a.n_seqs, a.q_stride}, {a.n_q_heads, a.q_head_stride}};
  return c.head_dim % 8 == 0 && divides(c.k, cache, 8) && divides(c.v, cache, 8) && divides(a.q, q, 8);
}

} // namespace

extern "C" {

int hf_append_kv(const hf_kv_cache *cache, const hf_append *args, void *hip_stream) {
  if (int rc = check_cache(cache)) return rc;
  if (!args) return set_error(HF_EINVAL, "null arguments");
  const hf_kv_cache &c = *cache;
  const hf_append &a = *args;
  if (a.n_tokens < 0) return set_error(HF_EINVAL, "negative size");
  if (a.flags & ~HF_ROT_INTERLEAVED) return set_error(HF_EINVAL, "unknown flag");
  if (a.rot_dim < 0 || a.rot_dim % 2 || a.rot_dim > c.head_dim) return set_error(HF_EINVAL, "rot_dim must be even and at most head_dim");
  if (!a.q != !a.q_out) return set_error(HF_EINVAL, "q and q_out go together");
  if (a.q && a.n_q_heads < 1) return set_error(HF_EINVAL, "n_q_heads must be positive");
  if (a.n_tokens == 0) return HF_OK;
  if (!a.k || !a.v || !a.slots) return set_error(HF_EINVAL, "null keys, values or slots");
  if (a.rot_dim && (!a.cos || !a.sin || !a.positions || a.n_positions < 1)) return set_error(HF_EINVAL, "a rotation needs cos, sin and positions");
  if (!aligned(a.q, 2) || !aligned(a.q_out, 2) || !aligned(a.k, 2) || !aligned(a.v, 2) || !aligned(a.slots, 8) || !aligned(a.cos, 4) ||
      !aligned(a.sin, 4) || !aligned(a.positions, 4))
    return set_error(HF_EINVAL, "arrays must be aligned to their elements");
  const Dim q[] = {{a.n_tokens, a.q_stride}, {a.n_q_heads, a.q_head_stride}}, q_out[] = {{a.n_tokens, a.q_out_stride}, {a.n_q_heads, a.q_out_head_stride}};
  const Dim k[] = {{a.n_tokens, a.k_stride}, {c.n_kv_heads, a.k_head_stride}}, v[] = {{a.n_tokens, a.v_stride}, {c.n_kv_heads, a.v_head_stride}};
  const Dim page[] = {{c.n_pages, c.page_stride}, {c.n_kv_heads, c.head_stride}, {c.page_tokens, c.token_stride}};
  if (!span(k, c.head_dim) || !span(v, c.head_dim)) return set_error(HF_EINVAL, "strides of keys or values are negative or span too much");
  if (a.q) {
    const int64_t in = span(q, c.head_dim), out = span(q_out, c.head_dim);
    if (!in || !out) return set_error(HF_EINVAL, "strides of queries are negative or span too much");
    if (!separate(q_out, c.head_dim)) return set_error(HF_EINVAL, "q_out overlaps itself");
    const bool same = a.q == a.q_out && (a.n_tokens == 1 || a.q_stride == a.q_out_stride) && (a.n_q_heads == 1 || a.q_head_stride == a.q_out_head_stride);
    if (!same && overlap(a.q, 2 * in, a.q_out, 2 * out)) return set_error(HF_EINVAL, "q_out overlaps q and is not q");
  }
  if ((uint64_t)a.n_tokens > hf::kMaxWgs) return set_error(HF_ERANGE, "too many tokens for one launch");
  int vec = 8;
  while (vec > 1 && (c.head_dim % vec || a.rot_dim % (2 * vec) || !divides(a.k, k, vec) || !divides(a.v, v, vec) || !divides(c.k, page, vec) ||
                     !divides(c.v, page, vec) || (a.q && (!divides(a.q, q, vec) || !divides(a.q_out, q_out, vec)))))
    vec /= 2;
  return launched(hf::launch_append(c, a, vec, hip_stream));
}

size_t hf_attend_workspace_bytes(const hf_kv_cache *cache, const hf_attention *args) {
  if (check_attention(cache, args)) return (size_t)-1;
  // the larger of what aligned and other tensors take: the pointers need not be known yet
  const size_t a = hf::attend_shape(*cache, *args, true).workspace, b = hf::attend_shape(*cache, *args, false).workspace;
  return a > b ? a : b;
}

int hf_attend(const hf_kv_cache *cache, const hf_attention *args, void *hip_stream) {
  if (int rc = check_attention(cache, args)) return rc;
  const hf_kv_cache &c = *cache;
  const hf_attention &a = *args;
  if (a.n_seqs == 0) return HF_OK;
  if (!a.q || !a.out || !a.suffix_lens || (a.suffix_width && !a.suffix_pages)) return set_error(HF_EINVAL, "null queries, output, lengths or pages");
  if (a.n_groups && (!a.group_offsets || !a.prefix_lens || (a.prefix_width && !a.prefix_pages)))
    return set_error(HF_EINVAL, "groups need their offsets, lengths and pages");
  if (!aligned(a.q, 2) || !aligned(a.out, 2) || !aligned(a.lse, 4) || !aligned(a.suffix_lens, 4) || !aligned(a.suffix_pages, 4) ||
      !aligned(a.group_offsets, 4) || !aligned(a.prefix_lens, 4) || !aligned(a.prefix_pages, 4))
    return set_error(HF_EINVAL, "arrays must be aligned to their elements");
  const Dim q[] = {{a.n_seqs, a.q_stride}, {a.n_q_heads, a.q_head_stride}}, out[] = {{a.n_seqs, a.out_stride}, {a.n_q_heads, a.out_head_stride}};
  const int64_t in = span(q, c.head_dim), to = span(out, c.head_dim);
  if (!in || !to) return set_error(HF_EINVAL, "strides of queries or output are negative or span too much");
  if (!separate(out, c.head_dim)) return set_error(HF_EINVAL, "the output overlaps itself");
  if (overlap(a.q, 2 * in, a.out, 2 * to)) return set_error(HF_EINVAL, "the output overlaps the queries");
  const bool vec = attention_vec(c, a);
  const hf::AttendLaunch shape = hf::attend_shape(c, a, vec);
  if (!shape.fits) return set_error(HF_ERANGE, "too much work for one launch");
  if (shape.workspace) {
    if (!a.workspace || !aligned(a.workspace, 16)) return set_error(HF_EINVAL, "the workspace must be given and 16-byte aligned");
    if (a.workspace_bytes < shape.workspace) return set_error(HF_EINVAL, "the workspace is smaller than hf_attend_workspace_bytes says");
  }
  return launched(hf::launch_attend(c, a, shape, vec, hip_stream));
}

int hf_token_logprobs(const hf_logits *in, const hf_logprobs *out, void *hip_stream) {
  if (int rc = check_logits(in)) return rc;
  if (!out) return set_error(HF_EINVAL, "null arguments");
  if (out->top_n < 0 || out->top_n > HF_MAX_TOP || out->top_n > in->vocab) return set_error(HF_EINVAL, "top_n must be in [0, min(vocab, HF_MAX_TOP)]");
  if (out->logprob && !in->targets) return set_error(HF_EINVAL, "log probabilities need targets");
  if (!aligned(out->logprob, 4) || !aligned(out->entropy, 4) || !aligned(out->lse, 4) || !aligned(out->norm, 4) || !aligned(out->top_ids, 4) || !aligned(out->top_logprobs, 4))
    return set_error(HF_EINVAL, "arrays must be aligned to their elements");
  if (in->rows == 0) return HF_OK;
  if ((uint64_t)in->rows > hf::kMaxWgs / 4) return set_error(HF_ERANGE, "too many rows for one launch"); // workgroups of up to 1024 lanes
  return launched(hf::launch_token_logprobs(*in, *out, hip_stream));
}

int hf_token_logprobs_back(const hf_logits *in, const hf_logprobs_grad *grad, void *hip_stream) {
  if (int rc = check_logits(in)) return rc;
  if (!grad) return set_error(HF_EINVAL, "null arguments");
  if (in->rows == 0) return HF_OK;
  const size_t size = in->dtype == HF_F32 ? 4 : 2;
  if (!in->targets || !grad->norm || !grad->dlogits) return set_error(HF_EINVAL, "null targets, norm or dlogits");
  if (grad->grad_entropy && !grad->entropy) return set_error(HF_EINVAL, "the entropy's gradient needs the entropy");
  if (!aligned(grad->norm, 4) || !aligned(grad->entropy, 4) || !aligned(grad->grad_logprob, 4) || !aligned(grad->grad_entropy, 4) || !aligned(grad->dlogits, size))
    return set_error(HF_EINVAL, "arrays must be aligned to their elements");
  const Dim from[] = {{in->rows, in->row_stride}}, to[] = {{in->rows, grad->dlogits_stride}};
  const int64_t out = span(to, in->vocab);
  if (!out) return set_error(HF_EINVAL, "dlogits_stride is negative or spans too much");
  if (!separate(to, in->vocab)) return set_error(HF_EINVAL, "dlogits overlaps itself");
  const bool same = in->logits == grad->dlogits && (in->rows == 1 || in->row_stride == grad->dlogits_stride);
  if (!same && overlap(in->logits, size * span(from, in->vocab), grad->dlogits, size * out))
    return set_error(HF_EINVAL, "dlogits overlaps the logits and is not the logits");
  if ((uint64_t)in->rows > hf::kMaxWgs || (uint64_t)in->rows * hf::logprob_back_segments(*in) > hf::kMaxWgs)
    return set_error(HF_ERANGE, "too many rows for one launch");
  return launched(hf::launch_token_logprobs_back(*in, *grad, hip_stream));
}

} // extern "C"
