// Attention of many rows over a block-scaled cache (gfx950; include/kvq.h states
// both): chunk queries and windows with more (query, head) rows of a kv head than
// the tiles of block_tiles.hip take, chunked prefill above all.
//
// The products are those of the tiles (S^T = K Q^T, O^T += V^T P^T, weights in hi + lo
// halves, a block's scales as factors of scores and weights).  Here a workgroup
// turns each 32-token block into halves once, in LDS, for all its waves of 32 rows:
// 16 bytes of codes a thread, 16 operands of 1 KB a block, four blocks in flight.
//
// What bounds it: the matrix cores (48 products of 16 cycles for a wave's block) and
// the vector unit (about 180 instructions, of which 16 exponentials of four times
// the cost) alike, so a wave runs both at once: while block i's weights are
// computed, the products of block i + 1's scores and block i - 1's values run.
// The reference of a row's exponents moves rarely; when it does, the accumulators
// take the change after the values' products that still belong to the old one.
// 1024 queries of 32 heads over 16384 tokens of 8 kv heads: 352 us, 760 TFLOP/s of the
// attention, 1.14 PFLOP/s of products with the weights' lower halves; the matrix cores
// are busy half of the time.  All 256 registers are taken and 6 to 12 spill.  The interleaving in hand-written order is worth 20 us, the
// barrier every second block 16; reads of the next block's operands before the barrier,
// with fewer waits, were slower (436), the compiler's own order too (456).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "block_ops.h"
#include "decode_common.h"
#include "kvq_internal.h"
#include "kvq_layout.h"
#include "mfma_common.h"

namespace kvq {
namespace {

using namespace dec;
using block_ops::f4_t;
using block_ops::h2_t;
using block_ops::h8_t;
using block_ops::u4_t;
using mfma_ops::mfma;

constexpr float kTop = 14.f;        // weights stay below 2^14 ...
constexpr float kHeadroom = 6.f;    // ... a new reference puts the largest at 2^8
constexpr float kNoScore = -1e30f;  // below any score

// Blocks in LDS: with eight waves (a workgroup per compute unit) a barrier every
// second block, so that waves come apart and one's products run beside another's weights.
template <int NW>
struct Operands {
  static constexpr int kSlots = NW == 8 ? 8 : 4, kAhead = NW == 8 ? 3 : 2;  // blocks written ahead
  u4_t op[kSlots][16][64];  // of a block: keys (token half, 32 channels), values (16 channels)
  uint32_t top[8];          // fp16 tail: the pattern of the largest of 16 channels' values
};

// A workgroup's blocks of one (sequence, kv head, group of rows).
struct Part {
  int si, h, rw, b0, b1, total, split;
};

// Codes of a block on their way to LDS: 16 bytes of keys or values (four waves: both).
template <int NW>
struct Staged {
  u4_t x[8 / NW];
};

// Nothing moves across: products and vector instructions stay in the order written, one
// beside the other.  (The compiler's own order, all products and then the weights, leaves
// the matrix cores idle half of the time.)
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// lo halves of two numbers whose hi halves are h: each instruction reads a half as it is.
__device__ __forceinline__ uint32_t low_halves(uint32_t h, float a, float b) {
  float x, y;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(x) : "v"(h), "v"(a));
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(y) : "v"(h), "v"(b));
  return mfma_ops::h2u((h2_t){(_Float16)x, (_Float16)y});
}

template <bool K8, bool V8, int NW>
__device__ __forceinline__ void attend_rows(const DecodeArgs& a, const Part& wk, Operands<NW>& sm) {
  constexpr int kSlots = Operands<NW>::kSlots, kAhead = Operands<NW>::kAhead;
  const DecodeSeq& S = a.seq[wk.si];
  const uint8_t* ring = a.arena + S.head0 + (uint64_t)wk.h * a.head_stride;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, blk = lane >> 4;
  const int inv = (65536 + a.gqh - 1) / a.gqh;
  const int gsh = __builtin_ctz(a.gk), bsh = gsh - 5;

  const int rg = wk.rw * NW + wv;  // this wave's row group of 32
  const bool active = rg < a.nrg;
  const int seen0 = S.L - a.nqry + 1;
  const RowBlocks rb = row_blocks(a.nqry, a.qpr * NW, S.L, S.Lq, gsh, a.window, a.sinks, wk.rw);
  // token of block b of the list
  auto place = [&](int b) {
    if (b >= rb.packed) return 32 * (b - rb.packed + rb.tail0);
    return 32 * (b + ((b >> bsh) < rb.groups.sink ? 0 : (rb.groups.first - rb.groups.sink) << bsh));
  };
  const int wave_first = active ? seen0 + min(rg * a.qpr, a.nqry - 1) : 0;
  const int wave_limit = active ? seen0 + min(rg * a.qpr + a.qpr - 1, a.nqry - 1) : 0;

  // rows 16 u + col of the row group: query operands, limits
  u4_t q[2][4];
  int lim[2];
  float ksc[2];
  size_t at[2];
  bool live[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    typedef u4_t u4_any __attribute__((aligned(4)));
    const int g = 16 * u + col, x = (g * inv) >> 16, j0 = rg * a.qpr + (x < a.qpr ? x : kSpareRow), j = min(j0, a.nqry - 1);
    live[u] = j0 < a.nqry;
    lim[u] = seen0 + j;
    at[u] = (size_t)j * a.hq + wk.h * a.gqh + (g - x * a.gqh);
    const uint16_t* qr = a.q + ((size_t)S.seq * a.nqry * a.hq + at[u]) * kHeadDim + 16 * blk;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) q[u][kb] = *reinterpret_cast<const u4_any*>(qr + 64 * (kb >> 1) + 8 * (kb & 1));
  }

  // ------------------------------------------------ blocks to LDS
  // (pages come by vector loads a block ahead of their codes', scales two ahead of use:
  // results arrive in the order asked for, and no block waits for its own)
  const bool paged = a.pm.table != nullptr;
  const uint8_t* head = a.arena + (paged ? a.pm.pool0 + (uint64_t)wk.h * a.pm.page_head_bytes : S.head0 + (uint64_t)wk.h * a.head_stride);
  const int32_t* table = a.pm.table + (size_t)S.seq * a.pm.max_pages;
  const int page_shift = paged ? a.pm.page_shift : 31, in_page = paged ? a.pm.page_tokens - 1 : 0x7FFFFFFF;
  const uint64_t page_bytes = paged ? a.pm.page_bytes : 0;
  int zero = 0;
  asm("" : "+v"(zero));  // (keeps the loads' addresses in vector registers)
  const int n = wv & 3;
  const uint32_t k_at = ((n >> 1) * 16 + col) * kHeadDim + (n & 1) * 64 + 16 * blk, v_at = n * 1024 + lane * 16;
  const bool key_wave = NW == 4 || wv < 4;
  const uint64_t code0 = key_wave ? region(a.kc) : region(a.vc), value0 = region(a.vc), scale0 = region(a.km);
  const uint32_t code_at = key_wave ? k_at : v_at;
  auto page_of = [&](int b) { return paged ? table[(place(b) >> page_shift) + zero] : 0; };
  auto load = [&](int b, int page, Staged<NW>& o) __attribute__((always_inline)) {
    const int in = place(b) & in_page;
    const uint8_t* seg = head + (uint64_t)(uint32_t)page * page_bytes + (size_t)in * kHeadDim;
    o.x[0] = *reinterpret_cast<const u4_t*>(seg + code0 + code_at);
    if constexpr (NW == 4) o.x[1] = *reinterpret_cast<const u4_t*>(seg + value0 + v_at);
  };
  auto load_scale = [&](int b, int page) __attribute__((always_inline)) {
    const int in = place(b) & in_page;
    return *reinterpret_cast<const float2*>(head + (uint64_t)(uint32_t)page * page_bytes + scale0 + (size_t)((in >> gsh) + zero) * 8);
  };
  const int op_at = key_wave ? (n >> 1) * 4 + 2 * (n & 1) : 8 + 2 * n;
  auto put = [&](int b, const Staged<NW>& o) __attribute__((always_inline)) {
    u4_t(*op)[64] = sm.op[b & (kSlots - 1)];
    auto put2 = [&](auto e4m3, int i, u4_t x) __attribute__((always_inline)) {
      op[i][lane] = __builtin_bit_cast(u4_t, block_ops::operand<decltype(e4m3)::value>(x[0], x[1]));
      op[i + 1][lane] = __builtin_bit_cast(u4_t, block_ops::operand<decltype(e4m3)::value>(x[2], x[3]));
    };
    using K = std::integral_constant<bool, K8>;
    using V = std::integral_constant<bool, V8>;
    if constexpr (NW == 4) {
      put2(K{}, op_at, o.x[0]);
      put2(V{}, 8 + 2 * n, o.x[1]);
    } else if constexpr (K8 == V8) {
      put2(K{}, op_at, o.x[0]);
    } else {
      if (key_wave) put2(K{}, op_at, o.x[0]);
      else put2(V{}, op_at, o.x[0]);
    }
  };
  // A block of the fp16 tail: raw halves; tokens past the sequence are zeros.
  auto put_tail = [&](int b) {
    u4_t(*op)[64] = sm.op[b & (kSlots - 1)];
    const int t0 = place(b);
    for (int w = wv; w < 8; w += NW) {
      const int mb = w >> 2, kb = w & 3, t = t0 + 16 * mb + col;
      u4_t k = {0u, 0u, 0u, 0u}, v = {0u, 0u, 0u, 0u};
      if (t < S.L)
        k = *reinterpret_cast<const u4_t*>(ring + region(a.tk) +
                                           ((size_t)(t % a.W) * kHeadDim + 64 * (kb >> 1) + 16 * blk + 8 * (kb & 1)) * 2);
      const uint16_t* rv = reinterpret_cast<const uint16_t*>(ring + region(a.tv)) + 16 * w + col;
      uint32_t top = 0u;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int tv = t0 + value_token(blk, e);
        const uint32_t x = tv < S.L ? rv[(size_t)(tv % a.W) * kHeadDim] : 0u;
        v[e >> 1] |= x << (16 * (e & 1));
        top = max(top, x & 0x7FFFu);
      }
      op[w][lane] = k;
      op[8 + w][lane] = v;
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, s));
      if (lane == 0) sm.top[w] = top;
    }
  };

  // ------------------------------------------------ rows
  float m[2] = {kNoScore, kNoScore}, l[2] = {0.f, 0.f};
  f4_t acc[2][8];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[u][t] = (f4_t){0.f, 0.f, 0.f, 0.f};

  auto read_keys = [&](int b, u4_t (&k)[8]) __attribute__((always_inline)) {
    const u4_t(*op)[64] = sm.op[b & (kSlots - 1)];
#pragma unroll
    for (int i = 0; i < 8; ++i) k[i] = op[i][lane];
  };
  auto score = [&](int i, const u4_t (&k)[8], f4_t (&d)[2][2]) __attribute__((always_inline)) {  // operand i: token half, 32 channels
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const f4_t c = i & 3 ? d[u][i >> 2] : (f4_t){0.f, 0.f, 0.f, 0.f};
      d[u][i >> 2] = mfma(__builtin_bit_cast(h8_t, k[i]), __builtin_bit_cast(h8_t, q[u][i & 3]), c);
    }
  };
  auto scores = [&](int b, f4_t (&d)[2][2]) __attribute__((always_inline)) {
    u4_t k[8];
    read_keys(b, k);
#pragma unroll
    for (int i = 0; i < 8; ++i) score(i, k, d);
  };
  const h8_t none = {0, 0, 0, 0, 0, 0, 0, 0};
  h8_t ph[2] = {none, none}, pl[2] = {none, none};  // weights of the block before
  auto value_op = [&](int b, int mb) __attribute__((always_inline)) { return sm.op[b & (kSlots - 1)][8 + mb][lane]; };
  auto values = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int mb = 0; mb < 8; ++mb) {
      const h8_t v8 = __builtin_bit_cast(h8_t, value_op(b, mb));
#pragma unroll
      for (int u = 0; u < 2; ++u) acc[u][mb] = mfma(v8, ph[u], acc[u][mb]);
#pragma unroll
      for (int u = 0; u < 2; ++u) acc[u][mb] = mfma(v8, pl[u], acc[u][mb]);
    }
  };
  auto mask = [&](int b, f4_t (&d)[2][2]) __attribute__((always_inline)) {
    const int t0 = place(b);
    if (t0 + 32 > wave_first || (t0 < wave_limit - a.window && t0 + 32 > a.sinks)) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int left = lim[u] - t0 - 4 * blk, from = max(lim[u] - a.window, 0) - t0 - 4 * blk, sunk = a.sinks - t0 - 4 * blk;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int i = 16 * (e >> 2) + (e & 3);
          float s = i < left && (i >= from || i < sunk) ? d[u][e >> 2][e & 3] : -__builtin_inff();
          asm volatile("" : "+v"(s));  // (a branch: blocks within every window pass it by)
          d[u][e >> 2][e & 3] = s;
        }
      }
    }
  };
  // A block's value scale enters its weights' exponent, p = 2^(score + log2 s_v - m): the
  // reference m goes by what a weight contributes, and numbers of any size keep their
  // bits next to others.  The sum of the weights takes it out again.  (Keys of zeros: their
  // scores are 0 at any scale, where a hidden token's is -inf.)
  float f[2], top[2], alpha[2], up;  // of the block at hand
  auto find_top = [&](int u, const f4_t (&d)[2][2], float2 scale) __attribute__((always_inline)) {
    f[u] = ksc[u] * (scale.x > 0.f ? scale.x : 1.f);
    const f4_t y = d[u][0], z = d[u][1];
    top[u] = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])));
    top[u] = fmaxf(fmaf(top[u], f[u], up), kNoScore);
  };
  // Rows above the limit move their references; whether any did.
  auto refer = [&]() __attribute__((always_inline)) -> bool {
    if (__builtin_amdgcn_ballot_w64(top[0] - m[0] > kTop || top[1] - m[1] > kTop) == 0) return false;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float t = fmaxf(top[u], __shfl_xor(top[u], 16));  // the row's maximum over its four lanes
      t = fmaxf(t, __shfl_xor(t, 32));
      const float mn = t - m[u] > kTop ? t + (kHeadroom - kTop) : m[u];
      alpha[u] = __builtin_amdgcn_exp2f(m[u] - mn);
      l[u] *= alpha[u];
      m[u] = mn;
    }
    return true;
  };
  auto rescale = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int t = 0; t < 8; ++t) acc[u][t] *= alpha[u];
  };

  // packed blocks.  (LDS of the part before is read: its last barrier is behind that.)
  const int b0 = wk.b0, pe = min(wk.b1, rb.packed);
  if (b0 < pe) {
    const int last = pe - 1;  // (past the last block: that one again, unused)
    auto scalar_page = [&](int b) { return __builtin_amdgcn_readfirstlane(page_of(min(b, last))); };
    Staged<NW> st;
    float2 c0, c1;
    int pages[2];  // of blocks b + 2 and, kAhead = 3, b + 3
    {
      Staged<NW> first[kAhead];
      int at[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) at[i] = scalar_page(b0 + i);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) load(min(b0 + i, last), at[i], first[i]);
      c0 = load_scale(b0, at[0]);
      c1 = load_scale(min(b0 + 1, last), at[1]);
      pages[0] = kAhead == 3 ? at[kAhead - 1] : scalar_page(b0 + 2);
      pages[1] = scalar_page(b0 + 3);
#pragma unroll
      for (int u = 0; u < 2; ++u) ksc[u] = a.qscale * block_ops::lift_query(q[u]);
      for (int i = threadIdx.x; i < 8 * 64; i += 64 * NW)  // the values before the first block: zeros, of weights 0
        sm.op[(b0 - 1) & (kSlots - 1)][8 + (i >> 6)][i & 63] = (u4_t){0u, 0u, 0u, 0u};
#pragma unroll
      for (int i = 0; i < kAhead; ++i) put(b0 + i, first[i]);
    }
    load(min(b0 + kAhead, last), pages[kAhead - 2], st);
    int page_next = page_of(min(b0 + kAhead + 1, last));
    __syncthreads();
    f4_t d0[2][2], d1[2][2];
    scores(b0, d0);
    // LDS holds b - 1 (values), b, b + 1 .. ; b + kAhead is written, the one after it asked for
    auto block = [&](int b, f4_t (&d)[2][2], f4_t (&next)[2][2]) __attribute__((always_inline)) {
      u4_t k[8], v[4];
      read_keys(b + 1, k);  // (past the last block: whatever LDS holds, unused)
      mask(b, d);
      // the next block's scores beside the staging and this one's maxima
      in_order();
      score(0, k, next);
      put(b + kAhead, st);
      in_order();
      score(1, k, next);
      const int page = __builtin_amdgcn_readfirstlane(page_next);
      page_next = page_of(min(b + kAhead + 2, last));
      const float2 scale = c0;
      up = block_ops::log_scale(scale.y);
      c0 = c1;
      in_order();
      score(2, k, next);
      c1 = load_scale(min(b + 2, last), pages[0]);
      pages[0] = kAhead == 3 ? pages[1] : page;
      pages[1] = page;
      in_order();
      score(3, k, next);
      load(min(b + kAhead + 1, last), page, st);
      in_order();
      score(4, k, next);
      find_top(0, d, scale);
      in_order();
      score(5, k, next);
      find_top(1, d, scale);
      in_order();
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = value_op(b - 1, i);
      score(6, k, next);
      score(7, k, next);
      const bool moved = refer();
      // the values of the block before beside this one's weights: four products, a pair of weights
      const float down = __builtin_amdgcn_exp2f(-up);
      const float bias[2] = {up - m[0], up - m[1]};
      float sum[2] = {0.f, 0.f};
      u4_t hw[2], lw[2];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int u = i >> 2, t = i & 3;
        const h8_t v8 = __builtin_bit_cast(h8_t, v[i & 3]);
        in_order();
        acc[0][i] = mfma(v8, ph[0], acc[0][i]);
        float x0 = fmaf(d[u][t >> 1][2 * (t & 1)], f[u], bias[u]), x1 = fmaf(d[u][t >> 1][2 * (t & 1) + 1], f[u], bias[u]);
        asm volatile("" : "+v"(x0), "+v"(x1));
        in_order();
        acc[1][i] = mfma(v8, ph[1], acc[1][i]);
        float p0 = __builtin_amdgcn_exp2f(x0);
        asm volatile("" : "+v"(p0));
        in_order();
        acc[0][i] = mfma(v8, pl[0], acc[0][i]);
        float p1 = __builtin_amdgcn_exp2f(x1);
        asm volatile("" : "+v"(p1));
        in_order();
        acc[1][i] = mfma(v8, pl[1], acc[1][i]);
        if (i < 4) v[i] = value_op(b - 1, i + 4);
        sum[u] += p0 + p1;
        uint32_t h = mfma_ops::h2u((h2_t){(_Float16)p0, (_Float16)p1});
        asm("" : "+v"(h));
        uint32_t low = low_halves(h, p0, p1);
        asm volatile("" : "+v"(low), "+v"(sum[u]));  // (here, not after the products)
        hw[u][t] = h;
        lw[u][t] = low;
      }
      in_order();
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        l[u] = fmaf(sum[u], down, l[u]);
        ph[u] = __builtin_bit_cast(h8_t, hw[u]);
        pl[u] = __builtin_bit_cast(h8_t, lw[u]);
      }
      if (moved) rescale();  // after the products that belong to the old references
    };
    for (int b = b0; b < pe; b += 2) {
      block(b, d0, d1);
      if (NW == 4) __syncthreads();
      if (b + 1 < pe) block(b + 1, d1, d0);
      __syncthreads();
    }
    values(pe - 1);
    __syncthreads();
  } else {
#pragma unroll
    for (int u = 0; u < 2; ++u) ksc[u] = a.qscale * block_ops::lift_query(q[u]);
  }
  // the fp16 tail's
  for (int b = max(b0, rb.packed); b < wk.b1; ++b) {
    put_tail(b);
    __syncthreads();
    f4_t d[2][2];
    scores(b, d);
    mask(b, d);
    // values enter times the power of two that puts the block's largest at 2^7 or above: out
    // of reach of subnormal halves, which lose bits in products, and no further, since what
    // values are larger than codes their weights are smaller, and lose bits beside packed
    // blocks (at 2^14: 6e-4 of a row's output beside a scale 2^15 times its own).  A block
    // of zeros stands as a packed one.
    uint32_t most = 0u;
#pragma unroll
    for (int w = 0; w < 8; ++w) most = max(most, sm.top[w]);
    const int lift = most == 0u ? block_ops::kZeros : max(block_ops::lift_of(most) - 7, 0);
    const float2 scale = make_float2(1.f, ldexpf(1.f, -lift));
    up = (float)-lift;
    find_top(0, d, scale);
    find_top(1, d, scale);
    if (refer()) rescale();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float sum = 0.f;
      u4_t hw, lw;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(d[u][t >> 1][2 * (t & 1)], f[u], up - m[u]));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(d[u][t >> 1][2 * (t & 1) + 1], f[u], up - m[u]));
        sum += p0 + p1;
        const block_ops::Halves h = block_ops::split(p0, p1);
        hw[t] = h.hi;
        lw[t] = h.lo;
      }
      l[u] = fmaf(sum, ldexpf(1.f, lift), l[u]);
      ph[u] = __builtin_bit_cast(h8_t, hw);
      pl[u] = __builtin_bit_cast(h8_t, lw);
    }
#pragma unroll
    for (int mb = 0; mb < 8; ++mb) {
      u4_t w = value_op(b, mb);
      block_ops::lift_halves(w, lift);
#pragma unroll
      for (int u = 0; u < 2; ++u) acc[u][mb] = mfma(__builtin_bit_cast(h8_t, w), ph[u], acc[u][mb]);
#pragma unroll
      for (int u = 0; u < 2; ++u) acc[u][mb] = mfma(__builtin_bit_cast(h8_t, w), pl[u], acc[u][mb]);
    }
    __syncthreads();
  }

  // rows to the output (one part) or records
  if (!active) return;
  typedef f4_t f4_any __attribute__((aligned(4)));
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    l[u] += __shfl_xor(l[u], 16);
    l[u] += __shfl_xor(l[u], 32);
    if (!live[u]) continue;
    if (S.nsplit == 1) {
      const float r = 1.f / l[u];
      float* o = a.out + ((size_t)S.seq * a.nqry * a.hq + at[u]) * kHeadDim + 4 * blk;
#pragma unroll
      for (int t = 0; t < 8; ++t) *reinterpret_cast<f4_any*>(o + 16 * t) = acc[u][t] * r;
    } else {
      float* rec = a.ws + ((size_t)(S.ws_base + wk.split) * a.hq * a.nqry + at[u]) * kRecFloats;
#pragma unroll
      for (int t = 0; t < 8; ++t) *reinterpret_cast<f4_t*>(rec + 4 + 16 * t + 4 * blk) = acc[u][t];
      if (blk == 0) {
        rec[0] = l[u] > 0.f ? m[u] : -__builtin_inff();
        rec[1] = l[u];
      }
      if (wk.b1 == wk.total) {  // a row group of fewer parts than the sequence's most ends with empty records
        for (int split = wk.split + 1; split < S.nsplit; ++split) {
          float* r = a.ws + ((size_t)(S.ws_base + split) * a.hq * a.nqry + at[u]) * kRecFloats;
#pragma unroll
          for (int t = 0; t < 8; ++t) *reinterpret_cast<f4_t*>(r + 4 + 16 * t + 4 * blk) = (f4_t){0.f, 0.f, 0.f, 0.f};
          if (blk == 0) {
            r[0] = -__builtin_inff();
            r[1] = 0.f;
          }
        }
      }
    }
  }
}

// The work of a launch is one list: of every sequence, kv head and group of 32 NW
// rows its blocks and a.extra_units units that stand for a part's begin and end.  A
// workgroup takes a.units_per_wg of them.
template <bool K8, bool V8, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void block_rows_kernel(DecodeArgs a) {
  __shared__ __attribute__((aligned(16))) Operands<NW> sm;
  const int per = a.units_per_wg, end = min((int)(blockIdx.x + 1) * per, a.total_wg), gsh = __builtin_ctz(a.gk);
  const int nrw = (a.nrg + NW - 1) / NW;
  for (int u = blockIdx.x * per; u < end;) {
    Part p;
    p.si = block_ops::sequence_of(a, u);
    const DecodeSeq& S = a.seq[p.si];
    p.h = (u - S.wg_begin) / S.nq;
    int begin = S.wg_begin + p.h * S.nq;  // S.nq: units of a kv head
    p.rw = 0;
    int units;
    for (;; ++p.rw) {
      p.total = row_blocks(a.nqry, a.qpr * NW, S.L, S.Lq, gsh, a.window, a.sinks, p.rw).total;
      units = p.total + a.extra_units;
      if (p.rw == nrw - 1 || u < begin + units) break;
      begin += units;
    }
    p.b0 = min(u - begin, p.total);
    p.b1 = min(end - begin, p.total);
    p.split = (int)blockIdx.x - begin / per;
    // (units past the blocks alone: nothing is left to do, and the blocks' end has
    // written the empty records)
    if (p.b0 < p.b1) attend_rows<K8, V8, NW>(a, p, sm);
    u = begin + units;
  }
}

template <bool K8, bool V8>
int launch_types(const DecodeArgs& a, int waves, void* stream) {
  const dim3 grid((unsigned)((a.total_wg + a.units_per_wg - 1) / a.units_per_wg));
  hipStream_t s = (hipStream_t)stream;
  if (waves == 8) hipLaunchKernelGGL((block_rows_kernel<K8, V8, 8>), grid, dim3(512), 0, s, a);
  else hipLaunchKernelGGL((block_rows_kernel<K8, V8, 4>), grid, dim3(256), 0, s, a);
  return (int)hipGetLastError();
}

}  // namespace

int launch_block_rows(const DecodeArgs& a, int type_k, int type_v, int waves, void* stream) {
  if (a.total_wg <= 0) return 0;
  if (type_k == kBlockE4M3)
    return type_v == kBlockE4M3 ? launch_types<true, true>(a, waves, stream) : launch_types<true, false>(a, waves, stream);
  return type_v == kBlockE4M3 ? launch_types<false, true>(a, waves, stream) : launch_types<false, false>(a, waves, stream);
}

}  // namespace kvq
