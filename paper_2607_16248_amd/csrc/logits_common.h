// Pieces shared by the kernels that read whole rows of logits in fp32, fp16 or
// bf16 (token sampling, the teacher loss): loads, sort keys, wave reductions.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

namespace kvq {
namespace logits {

// One type's storage and its value in fp32 (exact for all three).
struct F32 {
  typedef float raw;
  static __device__ __forceinline__ float value(raw x) { return x; }
  static __device__ __forceinline__ raw make(float x) { return x; }
};
struct F16 {
  typedef _Float16 raw;
  static __device__ __forceinline__ float value(raw x) { return (float)x; }
  static __device__ __forceinline__ raw make(float x) { return (_Float16)x; }
};
struct BF16 {
  typedef __bf16 raw;
  static __device__ __forceinline__ float value(raw x) { return (float)x; }
  static __device__ __forceinline__ raw make(float x) { return (__bf16)x; }
};

// 8 consecutive logits from p, which has its element's alignment only; those
// from `n` on read as -inf.
template <class T>
__device__ __forceinline__ void load8(const typename T::raw* p, int n, float (&v)[8]) {
  typedef typename T::raw vec __attribute__((ext_vector_type(8)));
  typedef vec vec_any __attribute__((aligned(sizeof(typename T::raw))));
  if (n >= 8) {
    const vec x = *reinterpret_cast<const vec_any*>(p);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = T::value(x[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? T::value(p[j]) : -__builtin_inff();
  }
}

// Keys whose order is that of (logit, lower index first): the sign-flipped bits
// of the fp32 value, then the complement of the index.
__device__ __forceinline__ uint32_t order_bits(float f) {
  const uint32_t u = __builtin_bit_cast(uint32_t, f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ uint64_t make_key(float v, uint32_t idx) {
  // (-0 and +0 are equal logits)
  return ((uint64_t)order_bits(v + 0.f) << 32) | (uint64_t)(~idx);
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __builtin_bit_cast(float, (o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return ~(uint32_t)k; }

__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int mask) {
  const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)v, mask), hi = (uint32_t)__shfl_xor((int)(uint32_t)(v >> 32), mask);
  return ((uint64_t)hi << 32) | lo;
}
__device__ __forceinline__ uint64_t shfl_up64(uint64_t v, int d) {
  const uint32_t lo = (uint32_t)__shfl_up((int)(uint32_t)v, d), hi = (uint32_t)__shfl_up((int)(uint32_t)(v >> 32), d);
  return ((uint64_t)hi << 32) | lo;
}
__device__ __forceinline__ uint64_t wave_max64(uint64_t v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint64_t o = shfl_xor64(v, d);
    v = o > v ? o : v;
  }
  return v;
}
__device__ __forceinline__ uint64_t wave_sum64(uint64_t v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += shfl_xor64(v, d);
  return v;
}
__device__ __forceinline__ uint64_t wave_scan64(uint64_t v) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint64_t o = shfl_up64(v, d);
    v += lane >= d ? o : 0;
  }
  return v;
}

}  // namespace logits
}  // namespace kvq
