// Pieces shared by the kernels that read whole rows of logits in fp32, fp16 or
// bf16 (token sampling, the teacher loss): loads, sort keys, wave reductions.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

namespace kvq {
namespace logits {

// One type's storage and its value in fp32 (exact for all three), whose lowest
// kZeroBits bits are zero.
struct F32 {
  typedef float raw;
  static constexpr int kZeroBits = 0;
  static __device__ __forceinline__ float value(raw x) { return x; }
  static __device__ __forceinline__ raw make(float x) { return x; }
};
struct F16 {
  typedef _Float16 raw;
  static constexpr int kZeroBits = 13;
  static __device__ __forceinline__ float value(raw x) { return (float)x; }
  static __device__ __forceinline__ raw make(float x) { return (_Float16)x; }
};
struct BF16 {
  typedef __bf16 raw;
  static constexpr int kZeroBits = 16;
  static __device__ __forceinline__ float value(raw x) { return (float)x; }
  static __device__ __forceinline__ raw make(float x) { return (__bf16)x; }
};

// 8 consecutive logits from p, which has its element's alignment only.
template <class T>
using raw8_t = typename T::raw __attribute__((ext_vector_type(8)));
template <class T>
__device__ __forceinline__ raw8_t<T> load8(const typename T::raw* p) {
  typedef raw8_t<T> any __attribute__((aligned(sizeof(typename T::raw))));
  return *reinterpret_cast<const any*>(p);
}
template <class T>
__device__ __forceinline__ raw8_t<T> all8(float x) {
  raw8_t<T> v;
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = T::make(x);
  return v;
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

// 64-bit wave reductions over DPP moves (no LDS round trips): shifts by 1, 2, 4
// and 8 within each row of 16 lanes, then the row totals through the row
// broadcasts 15 and 31.  Lanes without a source read 0.
template <int CTRL, int ROW_MASK = 0xF>
__device__ __forceinline__ uint64_t dpp64(uint64_t v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROW_MASK, 0xF, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROW_MASK, 0xF, false);
  return ((uint64_t)hi << 32) | lo;
}
__device__ __forceinline__ uint64_t lane64(uint64_t v, int lane) {
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}
__device__ __forceinline__ uint64_t wave_scan64(uint64_t v) {  // inclusive
  v += dpp64<0x111>(v);
  v += dpp64<0x112>(v);
  v += dpp64<0x114>(v);
  v += dpp64<0x118>(v);
  v += dpp64<0x142, 0xA>(v);
  v += dpp64<0x143, 0xC>(v);
  return v;
}
__device__ __forceinline__ uint64_t wave_sum64(uint64_t v) { return lane64(wave_scan64(v), 63); }

}  // namespace logits
}  // namespace kvq
