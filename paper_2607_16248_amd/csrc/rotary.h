// Rotation of queries and keys by their positions, as the append kernels apply it
// to the rows that they read (include/kvq.h, kvq_append_rotary):
//   a' = a cos - b sin,  b' = a sin + b cos
// for channels (a, b) of a pair.  Products of an fp16 (or bf16) number and an
// fp32 one are exact in fp64, so the sum is rounded there to 53 bits and once more
// to fp16: the quantizer that follows sees the numbers that the mathematics gives,
// and the bytes do not depend on how a compiler fuses.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "kvq_internal.h"

namespace kvq {
namespace rotary {

typedef uint32_t u4_t __attribute__((ext_vector_type(4)));
typedef float f4_t __attribute__((ext_vector_type(4)));
typedef f4_t f4_any __attribute__((aligned(4)));

__device__ __forceinline__ float from16(uint32_t bits, bool bf16) {
  return bf16 ? __builtin_bit_cast(float, bits << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}
__device__ __forceinline__ float lo16(uint32_t v, bool bf16) { return from16(v & 0xFFFFu, bf16); }
__device__ __forceinline__ float hi16(uint32_t v, bool bf16) { return from16(v >> 16, bf16); }

// Two fp32 numbers as fp16, rounded to nearest (v_cvt_pk of the default mode).
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)a) | ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)b) << 16);
}
// Inputs as fp16 numbers (exact for fp16; bf16 rounds below 2^-14 and overflows
// to infinity, which the packing reports).
__device__ __forceinline__ uint32_t to_half2(uint32_t v, bool bf16) {
  return bf16 ? pack16(lo16(v, true), hi16(v, true)) : v;
}

// d as an fp32 number that rounds to fp16 as d itself does.  Only an fp32 number
// on the border between two halves can go wrong: it takes its last bit from the
// side that d is on.
__device__ __forceinline__ float near_border(double d, float f) {
  const double back = (double)f;
  if (back == d) return f;
  const uint32_t u = __builtin_bit_cast(uint32_t, f);
  const bool further = __builtin_fabs(d) > __builtin_fabs(back);
  return __builtin_bit_cast(float, further ? u | 1u : (u - 1u) | 1u);
}
__device__ __forceinline__ bool on_border(float f) {
  const uint32_t u = __builtin_bit_cast(uint32_t, f) & 0x7FFFFFFFu;
  return (u & 0x1FFFu) == 0x1000u || (u < 0x38800000u && u != 0u);  // (subnormal halves: every number is looked at)
}

// Eight angles of a lane: pairs j0 .. j0 + 7 (neighbours: j0 .. j0 + 3).
struct Angles {
  double c[8], s[8];
};

// Channels 8 cc .. 8 cc + 7 of a row (16 lanes in a row of lanes hold one), whose
// angles are in g.  All 16 lanes are active.
struct Turn {
  int rot, half, cc;  // half: in lanes
  bool pairs, bf16, turns, second;
  int partner;        // lane of the other halves
  int j0;
  __device__ __forceinline__ Turn(const RotaryArgs& r, int lane) {
    rot = r.rot;
    pairs = r.pairs != 0;
    bf16 = r.bf16 != 0;
    cc = lane & 15;
    half = rot >> 4;
    turns = 8 * cc < rot;
    second = !pairs && cc >= half;
    partner = turns && !pairs ? (second ? lane - half : lane + half) : lane;
    j0 = pairs ? 4 * cc : 8 * (second ? cc - half : cc);
  }
  // position: a row of the tables
  __device__ __forceinline__ void load(const RotaryArgs& r, int64_t position, Angles& g) const {
    if (!turns) return;
    const float* c = r.cos_ + position * (rot >> 1) + j0;
    const float* s = r.sin_ + position * (rot >> 1) + j0;
    const f4_t c0 = *reinterpret_cast<const f4_any*>(c), s0 = *reinterpret_cast<const f4_any*>(s);
    f4_t c1 = c0, s1 = s0;
    if (!pairs) {
      c1 = *reinterpret_cast<const f4_any*>(c + 4);
      s1 = *reinterpret_cast<const f4_any*>(s + 4);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int n = e & 3;
      g.c[e] = e < 4 ? c0[n] : c1[n];
      g.s[e] = e < 4 ? s0[n] : s1[n];
    }
  }
  // the row's 8 channels x as rotated halves
  __device__ __forceinline__ u4_t apply(u4_t x, const Angles& g) const {
    u4_t y;
#pragma unroll
    for (int n = 0; n < 4; ++n) y[n] = (uint32_t)__shfl((int)x[n], partner);
    u4_t o;
#pragma unroll
    for (int n = 0; n < 4; ++n) o[n] = to_half2(x[n], bf16);
    if (!turns) return o;
    double d[8];
    if (pairs) {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const double a = lo16(x[n], bf16), b = hi16(x[n], bf16);
        d[2 * n] = __builtin_fma(a, g.c[n], -(b * g.s[n]));
        d[2 * n + 1] = __builtin_fma(a, g.s[n], b * g.c[n]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double own = e & 1 ? hi16(x[e >> 1], bf16) : lo16(x[e >> 1], bf16);
        const double other = e & 1 ? hi16(y[e >> 1], bf16) : lo16(y[e >> 1], bf16);
        const double t = other * g.s[e];
        d[e] = __builtin_fma(own, g.c[e], second ? t : -t);
      }
    }
    float f[8];
    bool any = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f[e] = (float)d[e];
      any |= on_border(f[e]);
    }
    if (__builtin_amdgcn_ballot_w64(any)) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (on_border(f[e])) f[e] = near_border(d[e], f[e]);
    }
#pragma unroll
    for (int n = 0; n < 4; ++n) o[n] = pack16(f[2 * n], f[2 * n + 1]);
    return o;
  }
};

// The table row of token i (of the call's) of a sequence, at place p of it.
__device__ __forceinline__ int64_t table_row(const RotaryArgs& r, uint8_t* arena, int64_t token, int p) {
  if (r.position == nullptr) return p;
  const int64_t at = r.position[token];
  if (at >= 0 && at < r.rows) return at;
  *reinterpret_cast<volatile uint32_t*>(arena) = 4u;  // KVQ_ERR_RANGE
  return 0;
}

// Eight elements of a row, 16 bytes at a time where rows allow it.
__device__ __forceinline__ u4_t load_row8(const uint16_t* p, bool aligned) {
  if (aligned) return *reinterpret_cast<const u4_t*>(p);
  u4_t v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (uint32_t)p[2 * i] | ((uint32_t)p[2 * i + 1] << 16);
  return v;
}

// The queries of tokens part * kQueryTokens .. of a sequence, heads of kv head h.
__device__ __forceinline__ void turn_queries(const AppendArgs& a, const RotaryArgs& r, const AppendSeq& S, int h, int part) {
  static_assert(kQueryTokens * 16 == kAppendThreads, "a lane per 8 channels of a token");
  typedef u4_t u4_any __attribute__((aligned(4)));
  const int i = part * kQueryTokens + (threadIdx.x >> 4);
  if (i >= S.L_new - S.L_old) return;
  const int64_t token = (int64_t)S.seq * a.n_max + i;
  const Turn turn(r, threadIdx.x & 63);
  Angles g;
  turn.load(r, table_row(r, a.arena, token, S.L_old + i), g);
  const uint16_t* in = r.q + token * r.q_stride + (int64_t)h * r.gqh * kHeadDim + 8 * turn.cc;
  uint16_t* out = r.q_out + ((token * a.hkv + h) * r.gqh) * kHeadDim + 8 * turn.cc;
  constexpr int kAhead = 4;
  for (int x0 = 0; x0 < r.gqh; x0 += kAhead) {
    u4_t q[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) q[u] = load_row8(in + min(x0 + u, r.gqh - 1) * kHeadDim, r.aligned != 0);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const u4_t o = turn.apply(q[u], g);
      if (x0 + u < r.gqh) *reinterpret_cast<u4_any*>(out + (x0 + u) * kHeadDim) = o;
    }
  }
}

}  // namespace rotary
}  // namespace kvq
