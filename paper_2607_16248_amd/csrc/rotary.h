// Rotation of queries and keys by their positions, as the append kernels apply it
// to the rows that they read (include/kvq.h, kvq_append_rotary):
//   a' = a cos - b sin,  b' = a sin + b cos
// for channels (a, b) of a pair, as if in 64 bits (products of an fp16 or bf16 number and
// an fp32 one are exact there) and rounded once to fp16: the quantizer that follows
// sees the numbers that the mathematics gives, and the bytes do not depend on how a
// compiler fuses.  Nearly all of them come from fp32 all the same: with q = fl(b sin)
// and its exact rest e (one fma), v = fl(fl(a cos - q) - e) is within 1.5 ulp of the
// exact sum, so its rounding to fp16 is right unless v lies within 2 ulp of the border
// of two halves (one number in 1600).  Those take the 64-bit way.  All in fp64, whose
// conversions run at a quarter of the rate: 16384 tokens of 32 query and 8 kv heads
// 164 us, 97 so; the bytes alone take 77 at a copy's rate.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "kvq_internal.h"

namespace kvq {
namespace rotary {

typedef uint32_t u4_t __attribute__((ext_vector_type(4)));
typedef float f4_t __attribute__((ext_vector_type(4)));
typedef f4_t f4_any __attribute__((aligned(4)));

// What a row holds (RotaryArgs::bf16), as the kernels' template argument.
enum Rows16 { kNone = 0, kHalf = 1, kBrain = 2 };

// Element e (0 or 1) of a pair.
template <int T>
__device__ __forceinline__ float at16(uint32_t v, int e) {
  if constexpr (T == kBrain) return __builtin_bit_cast(float, e ? v & 0xFFFF0000u : v << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(e ? v >> 16 : v));
}

// Two fp32 numbers as fp16, rounded to nearest (v_cvt_pk of the default mode).
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)a) | ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)b) << 16);
}
// Inputs as fp16 numbers (exact for fp16; bf16 rounds below 2^-14 and overflows
// to infinity, which is reported when it enters the cache).
template <int T>
__device__ __forceinline__ uint32_t to_half2(uint32_t v) {
  if constexpr (T == kBrain) return pack16(at16<T>(v, 0), at16<T>(v, 1));
  return v;
}

// Whether the number that v stands for may round to another half than v does: v within
// 2 ulp of a border of halves, among the subnormal ones, whose borders lie elsewhere, zero,
// whose sign the exact rest has covered, or not finite, which only the 64-bit way tells apart.
__device__ __forceinline__ bool near_border(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu;
  return ((u + 0x1002u) & 0x1FFFu) <= 4u || u < 0x38800000u || u >= 0x7F800000u;
}
// d as an fp32 number that rounds to fp16 as d itself does: where the conversion is not
// exact, its last bit says on which side of every border d is.
__device__ __forceinline__ float to_odd(double d) {
  const float f = (float)d;
  const double back = (double)f;
  if (back == d) return f;
  const uint32_t u = __builtin_bit_cast(uint32_t, f);
  return __builtin_bit_cast(float, __builtin_fabs(d) > __builtin_fabs(back) ? u | 1u : (u - 1u) | 1u);
}
// f[e] = x[e] c[e] + y[e] s[e], exact but for the one rounding that packs it.  near_border
// is tested over the eight at once (a border's distance is what the 19 low bits hold, and
// maximum passes a NaN on), and element by element only in waves where one failed: about
// every fourth.
__device__ __forceinline__ void turned(float (&f)[8], const float (&x)[8], const float (&c)[8], const float (&y)[8],
                                       const float (&s)[8]) {
  uint32_t border = ~0u;
  float least = __builtin_inff(), most = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float q = y[e] * s[e], rest = fmaf(y[e], s[e], -q);
    f[e] = fmaf(x[e], c[e], q) + rest;
    border = min(border, (__builtin_bit_cast(uint32_t, f[e]) << 19) + (0x1002u << 19));
    least = fminf(least, __builtin_fabsf(f[e]));
    most = __builtin_elementwise_maximum(most, __builtin_fabsf(f[e]));
  }
  if (__builtin_amdgcn_ballot_w64(border <= 4u << 19 || least < 0x1p-14f || !(most < __builtin_inff()))) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (near_border(f[e])) f[e] = to_odd(__builtin_fma((double)x[e], (double)c[e], (double)y[e] * (double)s[e]));
  }
}

// A lane's angles, by channel: a channel turns to x c + y s, y the other one of its pair.
struct Angles {
  float c[8], s[8];
};

// Channels 8 cc .. 8 cc + 7 of a row (16 lanes in a row of lanes hold one), whose
// angles are in g.  All 16 lanes are active.
template <int T>
struct Turn {
  int rot, half, cc;  // half: in lanes
  bool pairs, turns, second;
  int partner;        // lane of the other halves
  int j0;             // its first angle, of 8 (neighbours: of 4)
  __device__ __forceinline__ Turn(const RotaryArgs& r, int lane) {
    rot = r.rot;
    pairs = r.pairs != 0;
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
    if (pairs) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        g.c[e] = c0[e >> 1];
        g.s[e] = e & 1 ? s0[e >> 1] : -s0[e >> 1];
      }
    } else {
      const float sign = second ? 1.f : -1.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        g.c[e] = e < 4 ? c0[e & 3] : c1[e & 3];
        g.s[e] = sign * (e < 4 ? s0[e & 3] : s1[e & 3]);
      }
    }
  }
  // the row's 8 channels v as rotated halves
  __device__ __forceinline__ u4_t apply(u4_t v, const Angles& g) const {
    u4_t w, o;
#pragma unroll
    for (int n = 0; n < 4; ++n) w[n] = pairs ? __builtin_amdgcn_alignbit(v[n], v[n], 16) : (uint32_t)__shfl((int)v[n], partner);
#pragma unroll
    for (int n = 0; n < 4; ++n) o[n] = to_half2<T>(v[n]);
    if (!turns) return o;
    float x[8], y[8], f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = at16<T>(v[e >> 1], e & 1);
      y[e] = at16<T>(w[e >> 1], e & 1);
    }
    turned(f, x, g.c, y, g.s);
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

// Reports halves that are not finite (KVQ_ERR_RANGE).
__device__ __forceinline__ void report_range(uint8_t* arena, u4_t k, u4_t v) {
  typedef uint16_t us2_t __attribute__((ext_vector_type(2)));
  us2_t m = {0, 0};
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    m = __builtin_elementwise_max(m, __builtin_bit_cast(us2_t, k[n] & 0x7FFF7FFFu));
    m = __builtin_elementwise_max(m, __builtin_bit_cast(us2_t, v[n] & 0x7FFF7FFFu));
  }
  if (max(m.x, m.y) >= 0x7C00) *reinterpret_cast<volatile uint32_t*>(arena) = 4u;
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
template <int T>
__device__ __forceinline__ void turn_queries(const AppendArgs& a, const RotaryArgs& r, const AppendSeq& S, int h, int part) {
  static_assert(kQueryTokens * 16 == kAppendThreads, "a lane per 8 channels of a token");
  typedef u4_t u4_any __attribute__((aligned(4)));
  const int i = part * kQueryTokens + (threadIdx.x >> 4);
  if (i >= S.L_new - S.L_old) return;
  const int64_t token = (int64_t)S.seq * a.n_max + i;
  const Turn<T> turn(r, threadIdx.x & 63);
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
