// Launch interface between the C entry points of what surrounds a rollout's steps and their kernels.  Not part of the ABI.
// Every function expects arguments that its entry point has checked, never allocates or synchronises and returns a hipError_t value (0 = success).
#pragma once
#include <cstddef>
#include <cstdint>

#include "hfreshard.h"
#include "rollout_kernels.hpp" // enqueue_kernel, kMaxLanes, kMaxWgs

namespace hf {

// whether adjust_logits' workgroups fit a grid
bool adjust_fits(const hf_adjustment &args);
constexpr int32_t kMaxAdjustList = INT32_MAX - 511; // tokens or biases of a row
int launch_adjust(const hf_adjustment &args, void *stream);

int launch_top_distill(const hf_logits &in, const hf_distillation &args, void *stream);
int launch_top_distill_back(const hf_logits &in, const hf_distillation_grad &grad, void *stream);
// workgroups per row of top_distill_back
uint32_t distill_back_segments(const hf_logits &in);

size_t fork_workspace(const hf_page_pool &pool, const hf_page_fork &args);
size_t grow_workspace(const hf_page_pool &pool, const hf_page_grow &args);
size_t compact_workspace(const hf_page_pool &pool, const hf_page_compact &args);
int launch_fork(const hf_page_pool &pool, const hf_page_fork &args, void *stream);
int launch_grow(const hf_page_pool &pool, const hf_page_grow &args, void *stream);
int launch_compact(const hf_page_pool &pool, const hf_page_compact &args, void *stream);

} // namespace hf
