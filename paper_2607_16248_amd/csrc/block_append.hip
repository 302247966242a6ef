// Quantize-on-append for block-scaled caches (gfx950; include/kvq.h states the
// format): 8 bits an element, one fp32 scale of the keys and one of the values for
// each block of tokens and kv head,
//   s = fl(max |x| / top),  code = nearest number of the type to x / s, ties to even.
//
// One launch packs every block that leaves the fp16 window, copies the other new
// tokens into the ring and, in a rotated append, turns keys and queries (rotary.h).
// What bounds it: memory; a prefill reads 512 B of a token and kv head and writes
// 256, and its queries, where it has them, are twice that or more.  A workgroup of
// four waves takes a (sequence, kv head, block): it reads every element once into
// registers, the lanes as the packed caches' kernel (append.hip) has them, finds
// both maxima with one barrier, and packs.
// Codes are exact without a division.  Whole numbers: the rounded estimate f of x / s
// is right unless the estimate lies within 2^-13 of the middle of two (its error is
// below 2^-15); there d = x - f s, exact in one fma (f s has 31 bits, and |d| < s),
// against s / 2 says whether f or its neighbour is nearest.  e4m3: the hardware's
// conversion of the estimate is right unless that lies within 8 steps of fp32 from
// the middle of two numbers, or among the subnormal ones; there the sign of
// x - m s, m the middle, decides (exact: one fma).  A wave looks for such elements
// over eight at once.
// 8 kv heads, blocks of 128 whole numbers: 16384 tokens 32 us (3.1 TB/s), rotated 49, with
// 32 query heads 97 (3.9 TB/s).  A workgroup's loads, arithmetic and stores follow one
// another; a query workgroup has one pass of them, so nothing is asked for meanwhile.
// 4096 tokens in e4m3 blocks of 64: 25, 29 and 32 us, where the bytes take 19.
#include <hip/hip_runtime.h>

#include "append_common.h"
#include "decode_common.h"
#include "kvq_internal.h"
#include "kvq_layout.h"

namespace kvq {
namespace {

__device__ __forceinline__ float half_at(uint32_t v, int hi) {
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(hi ? v >> 16 : v));
}
// Larger magnitudes of two pairs of halves, as patterns (a NaN's or infinity's is
// 0x7C00 or more).
__device__ __forceinline__ uint32_t max_abs(uint32_t m, uint32_t x) {
  typedef uint16_t us2_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2_t, m),
                                                                __builtin_bit_cast(us2_t, x & 0x7FFF7FFFu)));
}

struct Scale {
  float s, rs;  // rs: about 1 / s; both 0 in a block without a finite scale or of zeros
};
// top: the pattern of the block's largest magnitude
__device__ __forceinline__ Scale scale_of(uint8_t* arena, uint32_t top, bool e4m3) {
  if (top >= 0x7C00u) {
    *reinterpret_cast<volatile uint32_t*>(arena) = 4u;  // KVQ_ERR_RANGE
    return {0.f, 0.f};
  }
  const float m = half_at(top, 0);
  if (m == 0.f) return {0.f, 0.f};
  const float s = m / (e4m3 ? 448.f : 127.f);
  return {s, __builtin_amdgcn_rcpf(s)};
}

// Number m (7 bits) of e4m3, the one past the largest (480) included.
__device__ __forceinline__ float e4m3_value(uint32_t m) {
  if (m < 8u) return (float)m * 0x1p-9f;
  return __builtin_bit_cast(float, (((m >> 3) + 120u) << 23) | ((m & 7u) << 20));
}

// Codes of eight elements (four pairs of halves), a byte each.
__device__ __forceinline__ uint2 whole_codes(const uint32_t (&x)[4], Scale g) {
  if (g.s == 0.f) return make_uint2(0x80808080u, 0x80808080u);
  constexpr float kWhole = 0x1.8p23f + 128.f;  // the sum's low byte: f + 128, f whole, ties to even
  uint32_t c[8];
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float y = half_at(x[e >> 1], e & 1) * g.rs, at = y + kWhole;
    most = fmaxf(most, __builtin_fabsf(y - (at - kWhole)));
    c[e] = __builtin_bit_cast(uint32_t, at);
  }
  if (__builtin_amdgcn_ballot_w64(most > 0.5f - 0x1p-13f)) {
    const float h = 0.5f * g.s;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = fmaf(kWhole - __builtin_bit_cast(float, c[e]), g.s, half_at(x[e >> 1], e & 1)), n = __builtin_fabsf(d);
      if (n > h || (n == h && (c[e] & 1u))) c[e] += d > 0.f ? 1u : ~0u;
    }
  }
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k)
    w[k] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[4 * k + 3], c[4 * k + 2], 0x0C0C0400u),
                                 __builtin_amdgcn_perm(c[4 * k + 1], c[4 * k], 0x0C0C0400u), 0x05040100u);
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint2 e4m3_codes(const uint32_t (&x)[4], Scale g) {
  if (g.s == 0.f) return make_uint2(0u, 0u);
  float y[8], least = __builtin_inff();
  uint32_t middle = ~0u;  // the low 20 bits of an estimate are its place between two numbers
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y[e] = half_at(x[e >> 1], e & 1) * g.rs;
    middle = min(middle, (__builtin_bit_cast(uint32_t, y[e]) << 12) + (0x80008u << 12));
    least = fminf(least, __builtin_fabsf(y[e]));
  }
  int w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    w[k] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k], y[4 * k + 1], 0, false);
    w[k] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k + 2], y[4 * k + 3], w[k], true);
  }
  if (__builtin_amdgcn_ballot_w64(middle <= 0x10u << 12 || least < 0x1p-6f)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int sh = 8 * (e & 3);
      const uint32_t code = ((uint32_t)w[e >> 2] >> sh) & 0xFFu, m = code & 0x7Fu;
      const float v = __builtin_fabsf(half_at(x[e >> 1], e & 1));
      const float at = e4m3_value(m), d = fmaf(-at, g.s, v);
      const uint32_t other = d > 0.f ? m + 1u : m - (m > 0u ? 1u : 0u);
      const float r = fmaf(-0.5f * (at + e4m3_value(other)), g.s, v);  // beyond the middle?
      const bool move = d > 0.f ? r > 0.f || (r == 0.f && (m & 1u)) : d < 0.f && (r < 0.f || (r == 0.f && (m & 1u)));
      if (move) w[e >> 2] = (int)(((uint32_t)w[e >> 2] & ~(0xFFu << sh)) | (((code & 0x80u) | other) << sh));
    }
  }
  return make_uint2((uint32_t)w[0], (uint32_t)w[1]);
}

template <int GK, bool AL, int ROT>
__device__ __forceinline__ void quantize_block(const AppendArgs& a, const RotaryArgs* rot, const AppendSeq& S, int h,
                                               int gi, bool k8, bool v8, uint32_t* tops) {
  const uint8_t* ring = a.arena + S.head0 + (uint64_t)h * a.head_stride;
  const int p0 = S.Lq_old + gi * GK;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cc = lane & 15, row = lane >> 4;
  const size_t token0 = (size_t)S.seq * a.n_max, ks = ROT ? rot->k_stride : (size_t)a.hkv * kHeadDim,
               vs = ROT ? rot->v_stride : (size_t)a.hkv * kHeadDim;
  const Rows rk{a.K + token0 * ks + (size_t)h * kHeadDim, reinterpret_cast<const uint16_t*>(ring + region(a.tk)), ks, S.L_old, a.W, p0 >= S.L_old};
  const Rows rv{a.V + token0 * vs + (size_t)h * kHeadDim, reinterpret_cast<const uint16_t*>(ring + region(a.tv)), vs, S.L_old, a.W, p0 >= S.L_old};
  u4_t kx[GK / 16];
#pragma unroll
  for (int i = 0; i < GK / 16; ++i) kx[i] = load8<AL>(rk.at(p0 + 16 * i + 4 * wv + row) + 8 * cc);
  uint32_t vx[GK / 32][8];
#pragma unroll
  for (int b = 0; b < GK / 32; ++b)
#pragma unroll
    for (int t = 0; t < 8; ++t) vx[b][t] = load2<AL>(rv.at(p0 + 32 * b + value_token(wv, t)) + 2 * lane);
  if constexpr (ROT) {
    const rotary::Turn<ROT> turn(*rot, lane);
#pragma unroll
    for (int i = 0; i < GK / 16; ++i) {
      const int p = p0 + 16 * i + 4 * wv + row;
      if (p < S.L_old) continue;  // (the ring's keys have turned; 16 lanes share a token)
      rotary::Angles g;
      turn.load(*rot, rotary::table_row(*rot, a.arena, (int64_t)(token0 + (p - S.L_old)), p), g);
      kx[i] = turn.apply(kx[i], g);
    }
    if constexpr (ROT == rotary::kBrain) {
#pragma unroll
      for (int b = 0; b < GK / 32; ++b)
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (p0 + 32 * b + value_token(wv, t) >= S.L_old) vx[b][t] = rotary::to_half2<ROT>(vx[b][t]);
    }
  }
  uint32_t mk = 0u, mv = 0u;
#pragma unroll
  for (int i = 0; i < GK / 16; ++i)
#pragma unroll
    for (int n = 0; n < 4; ++n) mk = max_abs(mk, kx[i][n]);
#pragma unroll
  for (int b = 0; b < GK / 32; ++b)
#pragma unroll
    for (int t = 0; t < 8; ++t) mv = max_abs(mv, vx[b][t]);
  // both as one pair, over the lanes and then the waves
  uint32_t top = max(mk & 0xFFFFu, mk >> 16) | (max(mv & 0xFFFFu, mv >> 16) << 16);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = max_abs(top, (uint32_t)__shfl_xor((int)top, d));
  if (lane == 0) tops[wv] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) top = max_abs(top, tops[w]);
  const Scale gk = scale_of(a.arena, top & 0xFFFFu, k8), gv = scale_of(a.arena, top >> 16, v8);

  int t0;
  uint8_t* seg = a.arena + packed_seg(a.pm, S.head0, a.head_stride, S.seq, h, p0, t0);
  if (threadIdx.x == 0) *reinterpret_cast<float2*>(seg + region(a.km) + (size_t)(t0 / GK) * 8) = make_float2(gk.s, gv.s);
  uint8_t* kd = seg + region(a.kc) + (size_t)t0 * kHeadDim;
#pragma unroll
  for (int i = 0; i < GK / 16; ++i) {
    const uint32_t x[4] = {kx[i][0], kx[i][1], kx[i][2], kx[i][3]};
    const uint2 w = k8 ? e4m3_codes(x, gk) : whole_codes(x, gk);
    *reinterpret_cast<uint2*>(kd + (size_t)(16 * i + 4 * wv + row) * kHeadDim + 8 * cc) = w;
  }
  // channels 2 lane and 2 lane + 1 of the wave's eight tokens: operand mb of lanes
  // c16 + 16 wv and the next (kvq_layout.h, block_value)
  const int mb = lane >> 3, c16 = 2 * (lane & 7);
  uint8_t* vd = seg + region(a.vc) + (size_t)t0 * kHeadDim + (mb >> 1) * 1024 + (c16 + 16 * wv) * 16 + 8 * (mb & 1);
#pragma unroll
  for (int b = 0; b < GK / 32; ++b) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      uint32_t x[4];
#pragma unroll
      for (int t = 0; t < 4; ++t)
        x[t] = __builtin_amdgcn_perm(vx[b][2 * t + 1], vx[b][2 * t], n ? 0x07060302u : 0x05040100u);
      const uint2 w = v8 ? e4m3_codes(x, gv) : whole_codes(x, gv);
      *reinterpret_cast<uint2*>(vd + (size_t)b * 4096 + 16 * n) = w;
    }
  }
}

template <int GK, bool AL, int ROT>
__device__ __forceinline__ void append_part(const AppendArgs& a, const RotaryArgs* rot, bool k8, bool v8) {
  __shared__ uint32_t tops[4];
  const int wg = blockIdx.x;
  const AppendSeq& S = a.seq[sequence_of(a, wg)];
  const int nquant = a.quantize ? S.n_quant : 0;
  int local = wg - S.wg_begin;
  if (local < nquant * a.hkv) {
    const PartHead q = part_head(local, nquant, a.hkv);
    quantize_block<GK, AL, ROT>(a, rot, S, q.h, q.part, k8, v8, tops);
  } else if (local -= nquant * a.hkv; !ROT || local < S.n_copy * a.hkv) {
    copy_ring<AL, ROT>(a, rot, S, local % a.hkv, local / a.hkv);
  } else if constexpr (ROT) {
    const PartHead q = part_head(local - S.n_copy * a.hkv, S.n_query, a.hkv);
    rotary::turn_queries<ROT>(a, *rot, S, q.h, q.part);
  }
}

template <int GK, bool AL>
__global__ __launch_bounds__(kAppendThreads) void append_block_kernel(AppendArgs a, bool k8, bool v8) {
  append_part<GK, AL, rotary::kNone>(a, nullptr, k8, v8);
}
template <int GK, bool AL, int ROT>
__global__ __launch_bounds__(kAppendThreads) void append_block_rotary_kernel(AppendArgs a, RotaryArgs rot, bool k8, bool v8) {
  append_part<GK, AL, ROT>(a, &rot, k8, v8);
}

template <int GK, bool AL>
int launch_blocks(const AppendArgs& a, const RotaryArgs* rot, bool k8, bool v8, hipStream_t s) {
  const dim3 grid(a.total_wg), block(kAppendThreads);
  if (rot == nullptr) hipLaunchKernelGGL((append_block_kernel<GK, AL>), grid, block, 0, s, a, k8, v8);
  else if (rot->bf16) hipLaunchKernelGGL((append_block_rotary_kernel<GK, AL, rotary::kBrain>), grid, block, 0, s, a, *rot, k8, v8);
  else hipLaunchKernelGGL((append_block_rotary_kernel<GK, AL, rotary::kHalf>), grid, block, 0, s, a, *rot, k8, v8);
  return (int)hipGetLastError();
}

}  // namespace

int launch_append_block(const AppendArgs& a, const RotaryArgs* rot, int type_k, int type_v, void* stream) {
  if (a.total_wg <= 0) return 0;
  const bool al = rot ? rot->aligned != 0 : (reinterpret_cast<uintptr_t>(a.K) | reinterpret_cast<uintptr_t>(a.V)) % 16 == 0;
  const bool k8 = type_k == kBlockE4M3, v8 = type_v == kBlockE4M3;
  hipStream_t s = (hipStream_t)stream;
  switch (a.gk) {
    case 32: return al ? launch_blocks<32, true>(a, rot, k8, v8, s) : launch_blocks<32, false>(a, rot, k8, v8, s);
    case 64: return al ? launch_blocks<64, true>(a, rot, k8, v8, s) : launch_blocks<64, false>(a, rot, k8, v8, s);
    case 128: return al ? launch_blocks<128, true>(a, rot, k8, v8, s) : launch_blocks<128, false>(a, rot, k8, v8, s);
    default: return (int)hipErrorInvalidValue;
  }
}

}  // namespace kvq
