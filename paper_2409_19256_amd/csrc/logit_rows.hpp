// Rows of logits as vectors of 16 bytes.  Device code only.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace hf {

template <typename T> constexpr int kVec = 16 / sizeof(T); // elements of a vector

// rows begin at any element, so the address of a vector is a multiple of the element's size and no more
template <typename T> struct Vector {
  typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
  typedef type any __attribute__((aligned(sizeof(T))));
};
template <typename T> __device__ __forceinline__ typename Vector<T>::type load_vec(const T *p) { return *reinterpret_cast<const typename Vector<T>::any *>(p); }
// what nobody reads again soon; it leaves the caches to others
template <typename T> __device__ __forceinline__ typename Vector<T>::type load_once(const T *p) { return __builtin_nontemporal_load(reinterpret_cast<const typename Vector<T>::any *>(p)); }
template <typename T> __device__ __forceinline__ void store_once(T *p, typename Vector<T>::type v) { __builtin_nontemporal_store(v, reinterpret_cast<typename Vector<T>::any *>(p)); }

// The larger ones; fmaxf would first make a quiet NaN of what might be a signalling one, an operation for every element.
__device__ __forceinline__ float larger(float a, float b) {
  float r;
  asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ float larger(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

} // namespace hf
