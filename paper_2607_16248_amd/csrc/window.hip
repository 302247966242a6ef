// Windowed attention of few rows (gfx950; include/kvq.h states it): up to 16
// (query, head) rows of a kv head over the key groups that their windows and the
// sinks touch, any bit class; errors of 2e-7 to 2e-6 against 64 bits.
//
// Every factor of both products is exact or carried to 22 bits: q as the fp16
// it is, keys and values as codes times scales in one or two halves (the
// operands of scaled_ops.h), weights p as hi + lo halves.  The products are
// transposed,
//   S^T = K' Q^T   (16 tokens x 16 rows; a lane holds 8 of its row's weights)
//   O^T = V'^T P^T (the same lanes' weights are the B operand),
// so a wave needs no LDS between them; zero-points enter as products of their
// own: K' Q^T with the group's z (and s) in every row gives sum_c q z in every
// lane, and z + c0 s of the value groups, in hi + lo halves, times P^T the value
// terms.
//
// A workgroup's four waves take key groups in turn (j0 + 4n of the split); a block's
// keys are asked for when the block before has its scores, its values when that
// block is done, and the page they lie in one block earlier: one set of registers
// that holds a block and, piece by piece, the next.  (Two whole sets, K2V2: the same
// loads in flight, 64 registers more, 20% slower; none, K8V8 over 8192 tokens: 303 us
// in one split, 130 so.)  One launch where a sequence has one split: its workgroup
// adds the fp16 tail and writes the output.
//
// What bounds it: the vector unit, by the unpacking, 3 instructions per pair of 1- and
// 2-bit elements and 4 of wider ones, about 400 per 32-token block with the softmax,
// beside 31 to 59 products; the widest classes the memory.  Measured, 8 kv heads: 32
// sequences, K8V8, five heads, 8192 tokens 130 us, 4.5 TB/s; four heads: 32 windows of
// 1024 K2V2 18 us, 64 of K4V4 31; one of 1024, K2V2, 14 us with its merge, which is
// two launches and their memory's latency.  With fields masked and moved into place
// apart, the hi halves converted twice and the masks of every block looked at, a block
// took 560 instructions (32 windows of 2048, K2V2: 26 us so, 31 then).  Tiles of two
// for 17 to 32 rows need 60 registers more than there are (five queries of four heads
// 42 us, in two row groups 27).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "decode_common.h"
#include "kvq_internal.h"
#include "kvq_layout.h"
#include "mfma_common.h"
#include "scaled_ops.h"
#include "tail_mfma.h"

namespace kvq {
namespace {

using namespace dec;
using namespace mfma_ops;

constexpr float kTop = 14.f;        // weights stay below 2^14 ...
constexpr float kHeadroom = 6.f;    // ... a new reference puts the largest at 2^8
constexpr float kNoScore = -1e30f;  // below any score
constexpr int kPartRows = 8;        // rows of one pass of the cross-wave reduction

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

// Masks of the code fields, kept in vector registers: a lane's field and the
// exponent above it then take one instruction (of three operands only one may be
// scalar).
template <int B>
struct Fields {
  static constexpr int n = B == 2 ? 4 : B == 4 ? 2 : 1;
  uint32_t m[n];
  __device__ __forceinline__ Fields() {
#pragma unroll
    for (int t = 0; t < n; ++t) {
      m[t] = B == 1 ? 0x80008000u : B == 2 ? 0x00030003u << (2 * t) : B == 4 ? 0x000F000Fu << (4 * t) : 0x64646464u;
      asm("" : "+v"(m[t]));
    }
  }
};

// (code - c0) / 2 of the codes at bits 2t (B == 2, t < 4) or 4t (B == 4, t < 2) of
// both halves of y, where they lie: with the exponent that gives the field's
// lowest bit the weight 1/2 (1) of its place, less that number and c0 / 2.
template <int B>
__device__ __forceinline__ h2_t field(uint32_t y, int t, const Fields<B>& f) {
  if constexpr (B == 2) {  // 2^(9 - 2t) + code / 2
    const uint32_t one = 0x60006000u - 0x08000800u * t;
    const _Float16 c = (_Float16)(-(float)(512 >> (2 * t)) - 0.5f);
    return u2h((y & f.m[t]) | one) + (h2_t){c, c};
  } else {  // 2^(10 - 4t) + code
    const uint32_t one = 0x64006400u - 0x10001000u * t;
    const _Float16 c = (_Float16)(-(float)(512 >> (4 * t)) - 4.f);
    return __builtin_elementwise_fma(u2h((y & f.m[t]) | one), (h2_t){(_Float16)0.5f, (_Float16)0.5f}, (h2_t){c, c});
  }
}
// Operand parts of 8 elements, as unpack_scaled's (x, at, s) of keys; a value's
// scales come with its power of two.
template <int B, bool VALUE>
__device__ __forceinline__ void unpack(const uint32_t (&x)[2], u4_t s, int at, const Fields<B>& f, u4_t& hi, u4_t& lo) {
  if constexpr (B == 1) {
#pragma unroll
    for (int t = 0; t < 4; ++t) hi[t] = ((x[0] << (15 - at - t)) & f.m[0]) | s[t];
  } else if constexpr (B == 2 && !VALUE) {
    const uint32_t y = x[0] >> at;
#pragma unroll
    for (int t = 0; t < 4; ++t) hi[t] = h2u(field<2>(y, t, f) * u2h(s[t]));
  } else if constexpr (B == 2) {  // element pair t at 4t, 4t + 16
    const uint32_t v = at ? x[0] >> 16 : x[0] & 0xFFFFu, y = v | (v << 14), z = y >> 8;
#pragma unroll
    for (int t = 0; t < 4; ++t) hi[t] = h2u(field<2>(t < 2 ? y : z, 2 * (t & 1), f) * u2h(s[t]));
  } else if constexpr (B == 4) {
    const uint32_t z = x[0] >> 8;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      uint32_t h, l;
      put_product(field<4>(t < 2 ? x[0] : z, t & 1, f), s[t], h, l);
      hi[t] = h;
      lo[t] = l;
    }
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t) {  // 1024 + code
      const h2_t h = u2h(__builtin_amdgcn_perm(f.m[0], x[t >> 1], t & 1 ? 0x04030402u : 0x04010400u));
      uint32_t p, l;
      put_product(__builtin_elementwise_fma(h, (h2_t){(_Float16)0.5f, (_Float16)0.5f}, (h2_t){(_Float16)-576.f, (_Float16)-576.f}),
                  s[t], p, l);
      hi[t] = p;
      lo[t] = l;
    }
  }
}

// What a wave reads of one 32-token block: its keys and their group's scales and
// zeros, asked for when the block before has its scores, and its values and their
// meta, asked for when that block is done.  FINE: value groups of 8 or 16
// channels, a scale row per operand; else one per 32 channels.
template <int BK>
struct KeyBlock {
  uint32_t x[2][BK];
  u4_t s[4], z[4];
};
template <int BV, bool FINE>
struct ValueBlock {
  uint32_t x[2 * BV];
  u4_t s[FINE ? 8 : 4], zz, zs;
};

template <int BK, int BV, bool FINE>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void window_kernel(DecodeArgs a) {
  __shared__ __attribute__((aligned(16))) Reduce<kPartRows> red;
  __shared__ float zsh[kWaves][16][17];  // value zero-point terms: [group][row]
  const Work wk = find_work<true, true>(a);
  const DecodeSeq& S = a.seq[wk.si];
  const uint8_t* ring = a.arena + S.head0 + (uint64_t)wk.h * a.head_stride;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, blk = lane >> 4;
  const int rows = a.qpr * a.gqh;  // of the group
  const int inv = (65536 + a.gqh - 1) / a.gqh;
  const size_t rec_rows = (size_t)a.hq * a.nqry;

  // the waves' results of rows r0 .. r0 + 7, merged into records (a sequence of one
  // split: into the output; every row sees a token, l > 0)
  auto write_rows = [&](int r0) {
    for (int idx = threadIdx.x; idx < kPartRows * kHeadDim; idx += blockDim.x) {
      const int r = idx / kHeadDim, c = idx % kHeadDim, g = r0 + r;
      const int x = (g * inv) >> 16, j = wk.rg * a.qpr + x;
      if (g >= rows || j >= a.nqry) continue;
      float M = -__builtin_inff();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M = fmaxf(M, red.m[w][r]);
      float val = 0.f, l = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = red.m[w][r] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(red.m[w][r] - M);
        val = fmaf(f, red.acc[w][idx], val);
        l = fmaf(f, red.l[w][r], l);
      }
      const size_t row = (size_t)j * a.hq + wk.h * a.gqh + g - x * a.gqh;
      if (S.nsplit == 1) {
        a.out[((size_t)S.seq * rec_rows + row) * kHeadDim + c] = val / l;
      } else {
        float* rec = a.ws + ((size_t)(S.ws_base + wk.sp) * rec_rows + row) * kRecFloats;
        rec[4 + c] = val;
        if (c == 0) { rec[0] = M; rec[1] = l; }
      }
    }
  };

  const int seen0 = S.L - a.nqry + 1;
  const int first_limit = seen0 + min(wk.rg * a.qpr, a.nqry - 1);
  const int last_limit = seen0 + min(wk.rg * a.qpr + a.qpr - 1, a.nqry - 1);
  const int ng = kHeadDim / a.gv, gsh = __builtin_ctz(a.gk), bsh = gsh - 5;
  const WindowGroups wg = window_groups(first_limit, last_limit, S.Lq, gsh, a.window, a.sinks);
  const int gps = a.split_tokens >> gsh;
  const int j0 = wk.sp * gps + ((wv + 2 * ((int)blockIdx.x >> 8)) & (kWaves - 1)), jend = min(wg.count, wk.sp * gps + gps);
  const int nblocks = j0 < jend ? ((jend - j0 + kWaves - 1) / kWaves) << bsh : 0;
  auto token_of = [&](int i) {
    int j = j0 + kWaves * (i >> bsh);
    j += j < wg.sink ? 0 : wg.first - wg.sink;
    return (j << gsh) + ((i & ((1 << bsh) - 1)) << 5);
  };

  // The page of block i's tokens; paged or not, one scalar load (of any word, times
  // 0 bytes), asked for a block ahead of the loads that need it.
  typedef const __attribute__((address_space(4))) int32_t scalar_t;
  const bool paged = a.pm.table != nullptr;
  const uint8_t* head = a.arena + (paged ? a.pm.pool0 + (uint64_t)wk.h * a.pm.page_head_bytes : S.head0 + (uint64_t)wk.h * a.head_stride);
  scalar_t* table = (scalar_t*)(paged ? a.pm.table + (size_t)S.seq * a.pm.max_pages : reinterpret_cast<const int32_t*>(ring + region(a.vb)));
  const int page_shift = paged ? a.pm.page_shift : 31, in_page = paged ? a.pm.page_tokens - 1 : 0x7FFFFFFF;
  const uint64_t page_bytes = paged ? a.pm.page_bytes : 0;
  auto page_of = [&](int i) { return table[token_of(i) >> page_shift]; };

  int vgl[FINE ? 8 : 4];  // byte offset of each scale row's 8 tokens
#pragma unroll
  for (int n = 0; n < (FINE ? 8 : 4); ++n) vgl[n] = ((FINE ? 16 * n + col : 32 * n) / a.gv) * 64 + 16 * blk;
  const int zrow = col < ng ? col : 0;
  auto load_keys = [&](int i, int page, KeyBlock<BK>& o) __attribute__((always_inline)) {
    const int t = token_of(i) & in_page;
    const uint8_t* seg = head + (uint64_t)(uint32_t)page * page_bytes;
    const uint8_t* kr = seg + region(a.kc) + (size_t)t * 16 * BK + col * 16 * BK + blk * 4 * BK;
#pragma unroll
    for (int mb = 0; mb < 2; ++mb) {
      if constexpr (BK == 1) {
        o.x[mb][0] = *reinterpret_cast<const uint32_t*>(kr + mb * 256);
      } else if constexpr (BK == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(kr + mb * 512);
        o.x[mb][0] = v.x;
        o.x[mb][1] = v.y;
      } else {
#pragma unroll
        for (int w = 0; w < BK / 4; ++w) {
          const u4_t v = *reinterpret_cast<const u4_t*>(kr + mb * 256 * BK + 16 * w);
#pragma unroll
          for (int n = 0; n < 4; ++n) o.x[mb][4 * w + n] = v[n];
        }
      }
    }
    const uint8_t* km = seg + region(a.km) + (size_t)(t >> gsh) * 512 + 16 * blk;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      o.s[kb] = *reinterpret_cast<const u4_t*>(km + 64 * kb);
      o.z[kb] = *reinterpret_cast<const u4_t*>(km + 256 + 64 * kb);
    }
  };
  auto load_values = [&](int i, int page, ValueBlock<BV, FINE>& o) __attribute__((always_inline)) {
    const int t = token_of(i) & in_page;
    const uint8_t* seg = head + (uint64_t)(uint32_t)page * page_bytes;
    const uint8_t* vr = seg + region(a.vc) + (size_t)(t >> 5) * 512 * BV + lane * 8 * BV;
    if constexpr (BV == 1) {
      const uint2 v = *reinterpret_cast<const uint2*>(vr);
      o.x[0] = v.x;
      o.x[1] = v.y;
    } else {
#pragma unroll
      for (int w = 0; w < BV / 2; ++w) {
        const u4_t v = *reinterpret_cast<const u4_t*>(vr + 16 * w);
#pragma unroll
        for (int n = 0; n < 4; ++n) o.x[4 * w + n] = v[n];
      }
    }
    const uint8_t* vm = seg + region(a.vm) + (size_t)(t >> 5) * 128 * ng;
#pragma unroll
    for (int n = 0; n < (FINE ? 8 : 4); ++n) o.s[n] = *reinterpret_cast<const u4_t*>(vm + vgl[n]);
    o.zs = *reinterpret_cast<const u4_t*>(vm + zrow * 64 + 16 * blk);
    o.zz = *reinterpret_cast<const u4_t*>(vm + (ng + zrow) * 64 + 16 * blk);
  };
  KeyBlock<BK> key;
  ValueBlock<BV, FINE> val;
  int page = 0;
  if (nblocks > 0) {  // under way before the queries are here
    page = page_of(0);
    load_keys(0, page, key);
    load_values(0, page, val);
    page = page_of(min(1, nblocks - 1));
  }

  // row col of the group: its query operand and limit (rows past whole
  // queries, and queries past the last, repeat the last query)
  u4_t q[4];
  int lim;
  {
    typedef u4_t u4_any __attribute__((aligned(4)));
    const int x = (col * inv) >> 16, j = min(wk.rg * a.qpr + (x < a.qpr ? x : kSpareRow), a.nqry - 1);
    lim = seen0 + j;
    const uint16_t* qr = a.q + (((size_t)S.seq * a.nqry + j) * a.hq + wk.h * a.gqh + (col - x * a.gqh)) * kHeadDim + 8 * blk;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      q[kb] = *reinterpret_cast<const u4_any*>(qr + 32 * kb);
      if constexpr (BK == 1) q[kb] ^= 0x80008000u;  // -q: the code term's factor is negative
    }
  }

  const int X = value_shift<BV>(*reinterpret_cast<const uint32_t*>(ring + region(a.vb)) & 0xFFFFu);
  const h2_t lift_s = {(_Float16)ldexpf(1.f, X), (_Float16)ldexpf(1.f, X)};
  const Fields<BK> fk;
  Fields<BV> fv;
  if constexpr (BV == BK) fv = fk;  // (one set of registers)
  // raw = alpha sum q z + beta sum q s + sum q K', score = ksc raw (q as held)
  constexpr float kAlpha = BK == 1 ? -2.f : 0.5f, kBeta = BK == 1 ? -1.f : Code<BK>::c0 * 0.5f;
  const float ksc = (BK == 1 ? 0.5f : 2.f) * a.qscale;

  // Small key numbers lose bits: halves below 2^-14 in the products, scales below
  // 2^-13 already in their half and in the lo parts, about 2^-25 of the query for
  // each.  Under queries of 8 or more they enter lifted by 2^12, in products of
  // their own next to larger ones (under smaller queries they move a weight by
  // less than 3e-7): keys of 2^-18 under queries of 2^14 are off by 5e-4 without
  // it and 1e-6 with it.  Such queries take a loop of their own.
  constexpr uint32_t kTinyScale = 0x0800u;  // 2^-13
  auto any_half = [](uint32_t w, uint32_t from, uint32_t to) -> bool {  // of the wave's, in [from, to)
    return __builtin_amdgcn_ballot_w64((w & 0xFFFFu) - from < to - from || (w >> 16) - from < to - from) != 0;
  };

  float m = kNoScore, most = kNoScore, l = 0.f, zterm = 0.f;  // the row's reference, the lane's maximum
  f4_t acc[8], zal = {0.f, 0.f, 0.f, 0.f}, zar = {0.f, 0.f, 0.f, 0.f};  // value zero-point terms: lifted, as they are
#pragma unroll
  for (int t = 0; t < 8; ++t) acc[t] = (f4_t){0.f, 0.f, 0.f, 0.f};

  // s[e] + zterm / ksc: raw scores
  auto scores = [&](auto lift_c, int i, float (&s)[8]) __attribute__((always_inline)) {
    constexpr bool LIFT = decltype(lift_c)::value;
    const bool first = (i & ((1 << bsh) - 1)) == 0;  // of its key group
    // raw scores of the scales ks (the group's, or a part of them; the rest 0)
    auto raw_scores = [&](const u4_t (&ks)[4], f4_t (&d)[2]) __attribute__((always_inline)) {
#pragma unroll
      for (int mb = 0; mb < 2; ++mb) {
        d[mb] = (f4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
          uint32_t x[2];
          x[0] = key.x[mb][BK == 1 ? 0 : BK == 2 ? kb >> 1 : BK == 4 ? kb : 2 * kb];
          x[1] = BK == 8 ? key.x[mb][2 * kb + 1 < BK ? 2 * kb + 1 : 0] : 0u;
          u4_t hi, lo;
          unpack<BK, false>(x, ks[kb], BK == 1 ? 4 * kb : 8 * (kb & 1), fk, hi, lo);
          d[mb] = mfma(__builtin_bit_cast(h8_t, hi), __builtin_bit_cast(h8_t, q[kb]), d[mb]);
          if constexpr (Code<BK>::parts == 2)
            d[mb] = mfma(__builtin_bit_cast(h8_t, lo), __builtin_bit_cast(h8_t, q[kb]), d[mb]);
        }
      }
    };
    auto q_sum = [&](const u4_t (&x)[4]) {  // sum over the channels of q x, the same in every lane of the row
      f4_t t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) t = mfma(__builtin_bit_cast(h8_t, x[kb]), __builtin_bit_cast(h8_t, q[kb]), t);
      return t[0];
    };
    auto all_of = [&](const u4_t (&x)[4], uint32_t mask, uint32_t from, uint32_t to) {  // any of the group's halves in [from, to)
      bool any = false;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int n = 0; n < 4; ++n) any |= any_half(x[kb][n] & mask, from, to);
      return any;
    };
    f4_t d[2];
    if (LIFT && (all_of(key.s, ~0u, 1u, kTinyScale) || all_of(key.z, 0x7FFF7FFFu, 1u, 0x0400u))) {
      // the small numbers lifted, apart from the others
      u4_t part[4], rest[4];
      if (first) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            uint32_t x, y;
            split_subnormal(key.z[kb][n], x, y);
            part[kb][n] = x;
            rest[kb][n] = y;
          }
        zterm = kAlpha * ksc * fmaf(1.f / kLift, q_sum(rest), q_sum(part));
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = 0.f;
      auto add = [&](float f) __attribute__((always_inline)) {
        raw_scores(part, d);
        if (first) zterm = fmaf(kBeta * ksc * f, q_sum(part), zterm);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = fmaf(d[e >> 2][e & 3], f, s[e]);
      };
      auto keep = [&](bool small) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const uint32_t w = key.s[kb][n];
            const uint32_t lo = ((w & 0xFFFFu) < kTinyScale) == small ? 0xFFFFu : 0u, hi = ((w >> 16) < kTinyScale) == small ? 0xFFFF0000u : 0u;
            part[kb][n] = w & (lo | hi);
          }
      };
      if (all_of(key.s, ~0u, kTinyScale, 0x7FFFu)) {
        keep(false);
        add(1.f);
      }
      if (all_of(key.s, ~0u, 1u, kTinyScale)) {
        keep(true);
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) part[kb] = __builtin_bit_cast(u4_t, lifted(part[kb], false));
        add(1.f / kLift);
      }
    } else {
      if (first) zterm = fmaf(kAlpha, q_sum(key.z), kBeta * q_sum(key.s)) * ksc;
      raw_scores(key.s, d);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = d[e >> 2][e & 3];
    }
    const int tok = token_of(i);
    if (tok + 32 > first_limit || (tok < last_limit - a.window && tok + 32 > a.sinks)) {
      // token tok + 16mb + 4blk + r is visible below the limit, from the window's
      // begin on or below the sinks' end
      const int left = lim - tok - 4 * blk, from = max(lim - a.window, 0) - tok - 4 * blk, sunk = a.sinks - tok - 4 * blk;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int n = 16 * (e >> 2) + (e & 3);
        s[e] = n < left && (n >= from || n < sunk) ? s[e] : -__builtin_inff();
        asm volatile("" : "+v"(s[e]));  // (a branch: blocks within every window pass it by)
      }
    }
  };

  auto attend = [&](const float (&s)[8]) __attribute__((always_inline)) {
    float top = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    top = fmaf(top, ksc, zterm);
    most = fmaxf(most, top);
    if (__builtin_amdgcn_ballot_w64(top - m > kTop)) {
      // the row's maximum over its four lanes; rows above the limit move
      // their reference
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = top - m > kTop ? top + (kHeadroom - kTop) : m;
      const float alpha = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int t = 0; t < 8; ++t) acc[t] *= alpha;
      zal *= alpha;
      zar *= alpha;
    }
    const float zm = zterm - m;  // (a hidden token's score is -inf: weight 0)
    u4_t hw, lw;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(s[2 * t], ksc, zm)), p1 = __builtin_amdgcn_exp2f(fmaf(s[2 * t + 1], ksc, zm));
      l += p0 + p1;
      const Halves h = split(p0, p1);
      hw[t] = h.hi;
      lw[t] = h.lo;
    }
    const h8_t ph = __builtin_bit_cast(h8_t, hw), pl = __builtin_bit_cast(h8_t, lw);
    // z + c0 s of the value groups, in hi + lo halves (22 bits): lifted below 8,
    // as it is in an accumulator of its own from there on.  (z and s apart are
    // opposite and leave their rounding where the values average out: 1e-6 over
    // 512 tokens of equal weight, 2e-7 so.)
    auto add_mid = [&](const float (&x)[8], f4_t& sum) __attribute__((always_inline)) {
      u4_t hi, lo;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const Halves h = split(x[2 * t], x[2 * t + 1]);
        hi[t] = h.hi;
        lo[t] = h.lo;
      }
      sum = mfma(__builtin_bit_cast(h8_t, hi), ph, sum);
      sum = mfma(__builtin_bit_cast(h8_t, hi), pl, sum);
      sum = mfma(__builtin_bit_cast(h8_t, lo), ph, sum);
    };
    float mid[8], mtop = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const h2_t z = u2h(val.zz[t]) * (h2_t){(_Float16)kLift, (_Float16)kLift}, sc = u2h(val.zs[t]);
      mid[2 * t] = fmaf((float)sc.x, Code<BV>::c0 * kLift, (float)z.x);
      mid[2 * t + 1] = fmaf((float)sc.y, Code<BV>::c0 * kLift, (float)z.y);
      mtop = fmaxf(mtop, fmaxf(fabsf(mid[2 * t]), fabsf(mid[2 * t + 1])));
    }
    if (__builtin_amdgcn_ballot_w64(!(mtop < 8.f * kLift)) == 0) {
      add_mid(mid, zal);
    } else {
      float big[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const h2_t z = u2h(val.zz[e >> 1]), sc = u2h(val.zs[e >> 1]);
        const float x = fmaf((float)(e & 1 ? sc.y : sc.x), Code<BV>::c0, (float)(e & 1 ? z.y : z.x));
        const bool is_big = fabsf(x) >= 8.f;
        big[e] = is_big ? x : 0.f;
        mid[e] = is_big ? 0.f : x * kLift;
      }
      add_mid(mid, zal);
      add_mid(big, zar);
    }
    u4_t vs;
#pragma unroll
    for (int mb = 0; mb < 8; ++mb) {
      uint32_t x[2];
      x[0] = val.x[BV == 1 ? mb >> 2 : BV == 2 ? mb >> 1 : BV == 4 ? mb : 2 * mb];
      x[1] = BV == 8 ? val.x[2 * mb + 1 < 2 * BV ? 2 * mb + 1 : 0] : 0u;
      if (FINE || mb % 2 == 0) {
#pragma unroll
        for (int t = 0; t < 4; ++t) vs[t] = h2u(u2h(val.s[FINE ? mb : mb >> 1][t]) * lift_s);
      }
      u4_t hi, lo;
      unpack<BV, true>(x, vs, BV == 1 ? 4 * (mb & 3) : 16 * (mb & 1), fv, hi, lo);
      acc[mb] = mfma(__builtin_bit_cast(h8_t, hi), ph, acc[mb]);
      acc[mb] = mfma(__builtin_bit_cast(h8_t, hi), pl, acc[mb]);
      if constexpr (Code<BV>::parts == 2) {
        acc[mb] = mfma(__builtin_bit_cast(h8_t, lo), ph, acc[mb]);
        acc[mb] = mfma(__builtin_bit_cast(h8_t, lo), pl, acc[mb]);
      }
    }
  };

  auto run = [&](auto lift_c) __attribute__((always_inline)) {
    const int last = nblocks - 1;
    for (int i = 0; i <= last; ++i) {
      float s[8];
      scores(lift_c, i, s);
      const int next = min(i + 1, last);  // (after the last block: that one again, unused)
      load_keys(next, page, key);
      attend(s);
      load_values(next, page, val);
      page = page_of(min(i + 2, last));
    }
  };
  if (nblocks > 0) {
    uint32_t qtop = 0u;  // the tile's largest |q| (the lanes hold all of it)
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int n = 0; n < 4; ++n) qtop = max(qtop, max(q[kb][n] & 0x7FFFu, (q[kb][n] >> 16) & 0x7FFFu));
    if (__builtin_amdgcn_ballot_w64(qtop >= 0x4800u) != 0) run(std::true_type{});  // 8.0
    else run(std::false_type{});
  }

  // zero-point terms of group 4blk + r, row col, to the lanes of its channels
#pragma unroll
  for (int r = 0; r < 4; ++r) zsh[wv][4 * blk + r][col] = fmaf(zal[r], 1.f / kLift, zar[r]);
  wave_lds_sync();
  TailState<1> st;
  const float unit = Code<BV>::unit * ldexpf(1.f, -X);
  const int gvsh = __builtin_ctz(a.gv);
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  most = fmaxf(most, __shfl_xor(most, 16));
  most = fmaxf(most, __shfl_xor(most, 32));
  const float to_max = __builtin_amdgcn_exp2f(m - most);  // records are relative to the maximum
  st.m[0] = l > 0.f ? most : -__builtin_inff();
  st.l[0] = l * to_max;
#pragma unroll
  for (int t = 0; t < 8; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int g = (FINE ? 16 * t + 4 * blk + r : 16 * t) >> gvsh;
      st.acc[0][t][r] = fmaf(acc[t][r], unit, zsh[wv][g][col]) * to_max;
    }
  if (S.L > S.Lq && wk.sp == S.nsplit - 1) {  // the fp16 tail: the last split's, or all of it
    TailState<1> tail;
    tail_split<1, 16, true, 4, true>(a, S, wk.h, wk.rg, ring, tail, lane, wv);
    const float top = fmaxf(st.m[0], tail.m[0]);  // (-inf in a wave that read nothing)
    const float f = st.l[0] > 0.f ? __builtin_amdgcn_exp2f(st.m[0] - top) : 0.f;
    const float ft = tail.l[0] > 0.f ? __builtin_amdgcn_exp2f(tail.m[0] - top) : 0.f;
    st.m[0] = top;
    st.l[0] = st.l[0] * f + tail.l[0] * ft;
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) st.acc[0][t][r] = st.acc[0][t][r] * f + tail.acc[0][t][r] * ft;
  }
  for (int r0 = 0; r0 < rows; r0 += kPartRows) {
    __syncthreads();
    stage_tail<kPartRows, 1>(st, 0, r0, red, lane, wv);
    __syncthreads();
    write_rows(r0);
  }
}

template <int BK, int BV>
int launch_fine(const DecodeArgs& a, void* stream) {
  if (a.gv < 32)
    hipLaunchKernelGGL((window_kernel<BK, BV, true>), dim3(a.total_wg), dim3(64 * kWaves), 0, (hipStream_t)stream, a);
  else
    hipLaunchKernelGGL((window_kernel<BK, BV, false>), dim3(a.total_wg), dim3(64 * kWaves), 0, (hipStream_t)stream, a);
  return (int)hipGetLastError();
}

}  // namespace

// This source is compiled once per key width (KVQ_BK, set by the build).
template <>
int launch_window_class<KVQ_BK>(const DecodeArgs& a, int bv, void* stream) {
  switch (bv) {
    case 1: return launch_fine<KVQ_BK, 1>(a, stream);
    case 2: return launch_fine<KVQ_BK, 2>(a, stream);
    case 4: return launch_fine<KVQ_BK, 4>(a, stream);
    case 8: return launch_fine<KVQ_BK, 8>(a, stream);
    default: return (int)hipErrorInvalidValue;
  }
}

}  // namespace kvq
