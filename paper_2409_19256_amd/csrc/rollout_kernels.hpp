// Launch interface between the C entry points of the rollout operators and their kernels.  Not part of the ABI.
// Every function expects arguments that rollout_abi.hip has checked, never allocates or synchronises and returns a
// hipError_t value (0 = success).
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "hfreshard.h"

namespace hf {

// A launch that reports its own error, and not one that another call has left behind.
template <typename... P, typename... A> hipError_t enqueue_kernel(void (*kernel)(P...), dim3 grid, int threads, hipStream_t st, A... args) {
  const auto go = [&](P... p) {
    void *list[] = {const_cast<void *>(static_cast<const void *>(&p))...};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, dim3(threads), list, 0, st);
  };
  const hipError_t e = go(args...);
  if (e != hipSuccess) (void)hipGetLastError(); // it is reported here, not to whoever asks next
  return e;
}

// elements per access of append_kv: the widest (8, 4, 2, 1) that divides the head, half of the rotated part, every stride and address
int launch_append(const hf_kv_cache &cache, const hf_append &args, int vec, void *stream);

// How hf_attend cuts its work, from the bounds in the arguments alone.
struct AttendShape {
  int32_t max_prefix, max_suffix;     // tokens, cut to what the tables can name
  int32_t prefix_chunk, suffix_chunk; // tokens of one part, multiples of 128
  int32_t prefix_parts, suffix_parts; // parts of the longest prompt and response
  int32_t row_waves;                  // prompts with more than 16 rows to a KV head: wavefronts of a workgroup that have rows of their own (32 each); 0 = no such
  bool lanes;                         // pages too small (or tokens too far apart) for addresses that a wavefront shares
  int32_t prefix_blocks, suffix_blocks; // query blocks
  bool small;                         // a workgroup for a sequence and KV head, over prompt and response: one launch
  bool direct;                        // one part a row: no merge
  bool ordered;                       // the longest responses first
  bool brief;                         // a wavefront, not a workgroup, for a response and KV head
  bool together;                      // responses in the grid of the prompts with many rows
  uint64_t prefix_wgs, suffix_wgs;
  size_t workspace;
};
// and what only the host needs of it
struct AttendLaunch : AttendShape {
  int32_t merge_split; // teams of lanes that share a row's parts in the merge
  uint64_t merge_wgs;
  bool fits; // every launch into a grid of fewer than 2^32 threads
};
// vec: every address, stride and the head are multiples of 8 elements
AttendLaunch attend_shape(const hf_kv_cache &cache, const hf_attention &args, bool vec);
// vec: every address, stride and the head are multiples of 8 elements
int launch_attend(const hf_kv_cache &cache, const hf_attention &args, const AttendLaunch &shape, bool vec, void *stream);

int launch_token_logprobs(const hf_logits &in, const hf_logprobs &out, void *stream);
int launch_token_logprobs_back(const hf_logits &in, const hf_logprobs_grad &grad, void *stream);

constexpr uint64_t kMaxWgs = 0xFFFFFFFFull / 256; // a HIP grid holds fewer than 2^32 threads
// workgroups per row of token_logprobs_back
uint32_t logprob_back_segments(const hf_logits &in);

} // namespace hf
