// Operand helpers of the block-scaled caches' attention: codes of 8 bits to exact
// fp16 operands, queries lifted to full halves, the reference of the value scales.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "kvq_internal.h"
#include "mfma_common.h"

namespace kvq {
namespace block_ops {

using mfma_ops::f4_t;
using mfma_ops::h2_t;
using mfma_ops::h2u;
using mfma_ops::h8_t;
using mfma_ops::u2h;
using mfma_ops::u4_t;

// Eight codes (a byte each) as halves, exactly.  e4m3: the conversion instruction,
// two elements each; whole numbers (held plus 128): the byte below the exponent of
// 1024, less 1152, two instructions for two elements.
template <bool E4M3>
__device__ __forceinline__ h8_t operand(uint32_t lo, uint32_t hi) {
  u4_t w;
  if constexpr (E4M3) {
    w[0] = h2u(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false));
    w[1] = h2u(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true));
    w[2] = h2u(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false));
    w[3] = h2u(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true));
  } else {
    const h2_t c = {(_Float16)-1152.f, (_Float16)-1152.f};
    w[0] = h2u(u2h(__builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u)) + c);
    w[1] = h2u(u2h(__builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u)) + c);
    w[2] = h2u(u2h(__builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u)) + c);
    w[3] = h2u(u2h(__builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)) + c);
  }
  return __builtin_bit_cast(h8_t, w);
}

// Exponent of the power of two that puts a half of pattern `top` (a magnitude) at 2^14 or
// above: 0 .. 38.
__device__ __forceinline__ int lift_of(uint32_t top) {
  const int e = (int)(__builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)top)) >> 23) - 127;
  return top == 0u ? 0 : max(14 - e, 0);
}
// Halves times 2^up, at most 2^15 at a time.
__device__ __forceinline__ void lift_step(u4_t& w, int step) {
  const _Float16 f = __builtin_bit_cast(_Float16, (uint16_t)((step + 15) << 10));
#pragma unroll
  for (int n = 0; n < 4; ++n) w[n] = h2u(u2h(w[n]) * (h2_t){f, f});
}
__device__ __forceinline__ void lift_halves(u4_t& w, int up) {  // up: the wave's
  for (; up > 0; up -= 15) lift_step(w, min(up, 15));
}

// A row's query, times the power of two that puts its largest element at 2^14 or
// above (elements 2^-28 of that and smaller would be subnormal halves, whose
// products lose bits).  Returns the power's reciprocal.  The row's four lanes (16
// apart) hold all of it.
__device__ __forceinline__ float lift_query(u4_t (&q)[4]) {
  typedef uint16_t us2_t __attribute__((ext_vector_type(2)));
  us2_t m = {0, 0};
#pragma unroll
  for (int kb = 0; kb < 4; ++kb)
#pragma unroll
    for (int n = 0; n < 4; ++n) m = __builtin_elementwise_max(m, __builtin_bit_cast(us2_t, q[kb][n] & 0x7FFF7FFFu));
  uint32_t top = max((uint32_t)m.x, (uint32_t)m.y);
  top = max(top, (uint32_t)__shfl_xor((int)top, 16));
  top = max(top, (uint32_t)__shfl_xor((int)top, 32));
  int up = lift_of(top);
  const float back = ldexpf(1.f, -up);
  do {
    const int step = min(up, 15);
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) lift_step(q[kb], step);
    up -= step;
  } while (__builtin_amdgcn_ballot_w64(up > 0) != 0);
  return back;
}

// Two numbers as hi + lo halves (22 bits).  (A pair's hi halves are converted once:
// left to itself, the compiler converts each a second time for the differences.)
struct Halves {
  uint32_t hi, lo;
};
__device__ __forceinline__ Halves split(float a, float b) {
  Halves h;
  h.hi = h2u((h2_t){(_Float16)a, (_Float16)b});
  asm("" : "+v"(h.hi));
  const h2_t x = u2h(h.hi);
  h.lo = h2u((h2_t){(_Float16)fmaf((float)x.x, -1.f, a), (_Float16)fmaf((float)x.y, -1.f, b)});
  return h;
}

// log2 of a block's value scale.  A block of zeros contributes nothing, but its weights
// count: in a row's reference it stands as one of scale 2^-80 (the smallest real one is
// 2^-24 / 448), so that weights of a block of scale s keep their bits while the zeros'
// scores lie less than 80 + log2 s above theirs.  The sum of weights takes the power out
// again: up to 2^14 2^80 per token, in range for 2^31 tokens.
constexpr int kZeros = 80;
__device__ __forceinline__ float log_scale(float s) { return s > 0.f ? __builtin_amdgcn_logf(s) : -(float)kZeros; }

// The sequence that holds unit u (DecodeSeq::wg_begin: its first unit): the last one
// that begins at u or before.
__device__ __forceinline__ int sequence_of(const DecodeArgs& a, int u) {
  static_assert(kMaxSeqPerLaunch <= 64, "one lane per sequence");
  if (a.nseq == 1) return 0;
  const int lane = threadIdx.x & 63;
  const auto* args = (const DecodeArgs*)__builtin_amdgcn_kernarg_segment_ptr();  // (indexed by lane, `a` would be copied)
  const int begin = args->seq[min(lane, kMaxSeqPerLaunch - 1)].wg_begin;
  return __popcll(__builtin_amdgcn_ballot_w64(lane < a.nseq && begin <= u)) - 1;
}

__device__ __forceinline__ float uniform(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
}

}  // namespace block_ops
}  // namespace kvq
