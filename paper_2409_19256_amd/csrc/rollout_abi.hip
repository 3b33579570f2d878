// C entry points of the rollout operators (declarations and contracts: include/hfreshard.h): the checks of what they are given.
#include <hip/hip_runtime.h>

#include "checks.hpp"
#include "rollout_kernels.hpp"

// the Python binding mirrors these layouts field by field
static_assert(sizeof(hf_kv_cache) == 64 && sizeof(hf_append) == 152 && sizeof(hf_attention) == 152, "ABI struct layout");
static_assert(sizeof(hf_logits) == 48 && sizeof(hf_logprobs) == 56 && sizeof(hf_logprobs_grad) == 48, "ABI struct layout");

namespace {

using hf::set_error;
using namespace hf::check;

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
    if (!span(q, c.head_dim) || !span(q_out, c.head_dim)) return set_error(HF_EINVAL, "strides of queries are negative or span too much");
    if (!separate(q_out, c.head_dim)) return set_error(HF_EINVAL, "q_out overlaps itself");
  }
  {
    const bool same = a.q == a.q_out && (a.n_tokens == 1 || a.q_stride == a.q_out_stride) && (a.n_q_heads == 1 || a.q_head_stride == a.q_out_head_stride);
    const Place from = a.q ? place(a.q, q, c.head_dim, 2) : Place{}, to = a.q ? place(a.q_out, q_out, c.head_dim, 2) : Place{};
    if (!same && overlap(from, to)) return set_error(HF_EINVAL, "q_out overlaps q and is not q");
    const int64_t table = a.rot_dim ? (int64_t)a.n_positions * (a.rot_dim / 2) : 0;
    const Output outputs[] = {{"keys of the cache overlap an input", place(c.k, page, c.head_dim, 2)},
                              {"values of the cache overlap an input or its keys", place(c.v, page, c.head_dim, 2)},
                              {"q_out overlaps an input or the cache", to}};
    if (const char *what = first_overlap(outputs, {place(a.k, k, c.head_dim, 2), place(a.v, v, c.head_dim, 2), same ? Place{} : from, array(a.cos, table, 4),
                                                   array(a.sin, table, 4), array(a.positions, a.rot_dim ? a.n_tokens : 0, 4), array(a.slots, a.n_tokens, 8)}))
      return set_error(HF_EINVAL, what);
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
  if (!span(q, c.head_dim) || !span(out, c.head_dim)) return set_error(HF_EINVAL, "strides of queries or output are negative or span too much");
  if (!separate(out, c.head_dim)) return set_error(HF_EINVAL, "the output overlaps itself");
  const bool vec = attention_vec(c, a);
  const hf::AttendLaunch shape = hf::attend_shape(c, a, vec);
  if (!shape.fits) return set_error(HF_ERANGE, "too much work for one launch");
  if (shape.workspace) {
    if (!a.workspace || !aligned(a.workspace, 16)) return set_error(HF_EINVAL, "the workspace must be given and 16-byte aligned");
    if (a.workspace_bytes < shape.workspace) return set_error(HF_EINVAL, "the workspace is smaller than hf_attend_workspace_bytes says");
  }
  const Dim page[] = {{c.n_pages, c.page_stride}, {c.n_kv_heads, c.head_stride}, {c.page_tokens, c.token_stride}};
  const int64_t n = a.n_seqs, groups = a.n_groups;
  const Output outputs[] = {{"the output overlaps an input", place(a.out, out, c.head_dim, 2)},
                            {"lse overlaps an input or the output", array(a.lse, n * a.n_q_heads, 4)},
                            {"the workspace overlaps an input or an output", array(a.workspace, shape.direct ? 0 : (int64_t)shape.workspace, 1)}};
  if (const char *what = first_overlap(outputs, {place(a.q, q, c.head_dim, 2), place(c.k, page, c.head_dim, 2), place(c.v, page, c.head_dim, 2), array(a.suffix_lens, n, 4),
                                                 array(a.suffix_pages, n * a.suffix_width, 4), array(a.group_offsets, groups ? groups + 1 : 0, 4),
                                                 array(a.prefix_lens, groups, 4), array(a.prefix_pages, groups * a.prefix_width, 4)}))
    return set_error(HF_EINVAL, what);
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
  const Dim from[] = {{in->rows, in->row_stride}};
  const Output outputs[] = {{"logprob overlaps an input", array(out->logprob, in->rows, 4)},
                            {"entropy overlaps an input or another output", array(out->entropy, in->rows, 4)},
                            {"lse overlaps an input or another output", array(out->lse, in->rows, 4)},
                            {"norm overlaps an input or another output", array(out->norm, 2 * in->rows, 4)},
                            {"top_ids overlap an input or another output", array(out->top_ids, in->rows * out->top_n, 4)},
                            {"top_logprobs overlap an input or another output", array(out->top_logprobs, in->rows * out->top_n, 4)}};
  if (const char *what = first_overlap(outputs, {place(in->logits, from, in->vocab, in->dtype == HF_F32 ? 4 : 2), array(in->targets, in->rows, in->target_bytes)}))
    return set_error(HF_EINVAL, what);
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
  if (!span(to, in->vocab)) return set_error(HF_EINVAL, "dlogits_stride is negative or spans too much");
  if (!separate(to, in->vocab)) return set_error(HF_EINVAL, "dlogits overlaps itself");
  if ((uint64_t)in->rows > hf::kMaxWgs || (uint64_t)in->rows * hf::logprob_back_segments(*in) > hf::kMaxWgs)
    return set_error(HF_ERANGE, "too many rows for one launch");
  const bool same = in->logits == grad->dlogits && (in->rows == 1 || in->row_stride == grad->dlogits_stride);
  const Place logits = place(in->logits, from, in->vocab, size);
  const Output outputs[] = {{"dlogits overlaps an input and is not the logits", place(grad->dlogits, to, in->vocab, size)}};
  if (const char *what = first_overlap(outputs, {same ? Place{} : logits, array(in->targets, in->rows, in->target_bytes), array(grad->norm, 2 * in->rows, 4),
                                                 array(grad->grad_entropy ? grad->entropy : nullptr, in->rows, 4), array(grad->grad_logprob, in->rows, 4),
                                                 array(grad->grad_entropy, in->rows, 4)}))
    return set_error(HF_EINVAL, what);
  return launched(hf::launch_token_logprobs_back(*in, *grad, hip_stream));
}

} // extern "C"
