// Exchanges between the lanes of a wavefront that stay in registers.  Device code only.
#pragma once
#include <hip/hip_runtime.h>

namespace hf {

// x of a lane and of the lane 32 (16) further, in either order: the instruction exchanges the upper half (odd rows of 16) of one register with the
// lower half (even rows) of the other.  Written by hand because the compiler's builtin gives its first result for both; the two
// wait states are those it puts between a write of the operands and the exchange.
__device__ __forceinline__ void swap32(float &a, float &b) { asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b)); }
__device__ __forceinline__ void swap16(float &a, float &b) { asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b)); }

template <int kControl> __device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), kControl, 0xF, 0xF, true));
}

struct Max {
  static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); }
};
struct Sum {
  static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};

// over the four lanes that are 16 apart
template <typename Op> __device__ __forceinline__ float over_rows(float x) {
  float y = x;
  swap32(x, y);
  x = y = Op::of(x, y);
  swap16(x, y);
  return Op::of(x, y);
}
// over the whole wavefront: lanes 1 and 2 apart, then mirrored in 8 and in 16, then the rows
template <typename Op> __device__ __forceinline__ float over_wave(float x) {
  x = Op::of(x, dpp<0xB1>(x));
  x = Op::of(x, dpp<0x4E>(x));
  x = Op::of(x, dpp<0x141>(x));
  x = Op::of(x, dpp<0x140>(x));
  return over_rows<Op>(x);
}

} // namespace hf
