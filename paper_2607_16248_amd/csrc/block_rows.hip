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

constexpr float kTop = 13.f;        // weights stay below 2^13, times a scale ratio up to 4
constexpr float kHeadroom = 6.f;    // a new reference puts the largest 2^7 below that
constexpr float kNoScore = -1e30f;  // below any score
constexpr int kSlots = 4;           // blocks in LDS

struct Operands {
  u4_t op[kSlots][16][64];    // of a block: keys (token half, 32 channels), values (16 channels)
  float2 scale[kSlots];
  uint32_t big[kSlots][8];    // fp16 tail: whether any value of 16 channels is 8 or more
};

// A workgroup's blocks of one (sequence, kv head, group of rows).
struct Part {
  int si, h, rw, b0, b1, total, split;
};

// Codes of a block on their way to LDS: 16 bytes of keys or values (four waves: both).
template <int NW>
struct Staged {
  u4_t x[8 / NW];
  float2 scale;
};

template <bool K8, bool V8, int NW>
__device__ __forceinline__ void attend_rows(const DecodeArgs& a, const Part& wk, Operands& sm) {
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
  const bool paged = a.pm.table != nullptr;
  auto load = [&](int b, Staged<NW>& o) __attribute__((always_inline)) {
    const int t = place(b);
    int in;
    const uint8_t* seg = a.arena + packed_seg(a.pm, S.head0, a.head_stride, S.seq, wk.h, t, in);
    const uint8_t* kr = seg + region(a.kc) + (size_t)in * kHeadDim;
    const uint8_t* vr = seg + region(a.vc) + (size_t)in * kHeadDim;
    const int n = wv & 3;
    const uint32_t k_at = ((n >> 1) * 16 + col) * kHeadDim + (n & 1) * 64 + 16 * blk, v_at = n * 1024 + lane * 16;
    if constexpr (NW == 8) {
      o.x[0] = *reinterpret_cast<const u4_t*>(wv < 4 ? kr + k_at : vr + v_at);
    } else {
      o.x[0] = *reinterpret_cast<const u4_t*>(kr + k_at);
      o.x[1] = *reinterpret_cast<const u4_t*>(vr + v_at);
    }
    o.scale = *reinterpret_cast<const float2*>(seg + region(a.km) + (size_t)(in >> gsh) * 8);
  };
  auto put = [&](int b, const Staged<NW>& o) __attribute__((always_inline)) {
    const int slot = b & (kSlots - 1), n = wv & 3;
    u4_t(*op)[64] = sm.op[slot];
    auto put_keys = [&](u4_t x) {
      op[(n >> 1) * 4 + 2 * (n & 1)][lane] = __builtin_bit_cast(u4_t, block_ops::operand<K8>(x[0], x[1]));
      op[(n >> 1) * 4 + 2 * (n & 1) + 1][lane] = __builtin_bit_cast(u4_t, block_ops::operand<K8>(x[2], x[3]));
    };
    auto put_values = [&](u4_t x) {
      op[8 + 2 * n][lane] = __builtin_bit_cast(u4_t, block_ops::operand<V8>(x[0], x[1]));
      op[8 + 2 * n + 1][lane] = __builtin_bit_cast(u4_t, block_ops::operand<V8>(x[2], x[3]));
    };
    if constexpr (NW == 8) {
      if (wv < 4) put_keys(o.x[0]);
      else put_values(o.x[0]);
    } else {
      put_keys(o.x[0]);
      put_values(o.x[1]);
    }
    if (threadIdx.x == 0) sm.scale[slot] = o.scale;
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
      const bool big = __builtin_amdgcn_ballot_w64(top >= 0x4800u) != 0;  // 8.0
      if (lane == 0) sm.big[b & (kSlots - 1)][w] = big;
    }
  };

  // ------------------------------------------------ rows
  float m[2] = {kNoScore, kNoScore}, l[2] = {0.f, 0.f};
  f4_t acc[2][8];
  block_ops::ValueUnit unit;
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[u][t] = (f4_t){0.f, 0.f, 0.f, 0.f};

  auto scores = [&](int b, f4_t (&d)[2][2]) __attribute__((always_inline)) {
    const u4_t(*op)[64] = sm.op[b & (kSlots - 1)];
#pragma unroll
    for (int mb = 0; mb < 2; ++mb) {
#pragma unroll
      for (int u = 0; u < 2; ++u) d[u][mb] = (f4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        const h8_t k8 = __builtin_bit_cast(h8_t, op[mb * 4 + kb][lane]);
#pragma unroll
        for (int u = 0; u < 2; ++u) d[u][mb] = mfma(k8, __builtin_bit_cast(h8_t, q[u][kb]), d[u][mb]);
      }
    }
  };
  const h8_t none = {0, 0, 0, 0, 0, 0, 0, 0};
  h8_t ph[2] = {none, none}, pl[2] = {none, none};  // weights of the block before
  auto values = [&](int b) __attribute__((always_inline)) {
    const u4_t(*op)[64] = sm.op[b & (kSlots - 1)];
#pragma unroll
    for (int mb = 0; mb < 8; ++mb) {
      const h8_t v8 = __builtin_bit_cast(h8_t, op[8 + mb][lane]);
#pragma unroll
      for (int u = 0; u < 2; ++u) acc[u][mb] = mfma(v8, ph[u], acc[u][mb]);
#pragma unroll
      for (int u = 0; u < 2; ++u) acc[u][mb] = mfma(v8, pl[u], acc[u][mb]);
    }
  };
  // The tail's values: lifted by 2^12 while all are below 8, else their normal halves
  // as they are and the subnormal ones lifted (products of those lose bits).
  auto tail_values = [&](int b) {
    const u4_t(*op)[64] = sm.op[b & (kSlots - 1)];
#pragma unroll
    for (int mb = 0; mb < 8; ++mb) {
      const u4_t w = op[8 + mb][lane];
      const bool big = sm.big[b & (kSlots - 1)][mb] != 0;
      u4_t normal = {0u, 0u, 0u, 0u}, lifted;
      if (big) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          uint32_t x, y;
          mfma_ops::split_subnormal(w[t], x, y);
          normal[t] = x;
          lifted[t] = y;
        }
      } else {
        lifted = __builtin_bit_cast(u4_t, mfma_ops::lifted(w, false));
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f4_t x = {0.f, 0.f, 0.f, 0.f};
        x = mfma(__builtin_bit_cast(h8_t, lifted), ph[u], x);
        x = mfma(__builtin_bit_cast(h8_t, lifted), pl[u], x);
        acc[u][mb] = mfma(__builtin_bit_cast(h8_t, normal), ph[u], acc[u][mb]);
        acc[u][mb] = mfma(__builtin_bit_cast(h8_t, normal), pl[u], acc[u][mb]);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[u][mb][r] = fmaf(x[r], 1.f / mfma_ops::kLift, acc[u][mb][r]);
      }
    }
  };

  // Scores d of block b to weights; `after` (products of other blocks that need
  // neither) runs beside the maxima, `before` beside the exponentials.
  auto softmax = [&](int b, f4_t (&d)[2][2], float s_k, float s_v, auto after, auto before) __attribute__((always_inline)) {
    const int t0 = place(b);
    if (t0 + 32 > wave_first || (t0 < wave_limit - a.window && t0 + 32 > a.sinks)) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int left = lim[u] - t0 - 4 * blk, from = max(lim[u] - a.window, 0) - t0 - 4 * blk, sunk = a.sinks - t0 - 4 * blk;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int n = 16 * (e >> 2) + (e & 3);
          float s = n < left && (n >= from || n < sunk) ? d[u][e >> 2][e & 3] : -__builtin_inff();
          asm volatile("" : "+v"(s));  // (a branch: blocks within every window pass it by)
          d[u][e >> 2][e & 3] = s;
        }
      }
    }
    after();
    float f[2], top[2], alpha[2] = {1.f, 1.f};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f[u] = ksc[u] * (s_k > 0.f ? s_k : 1.f);  // (a block of zeros has scores 0 at any scale; a hidden token's is -inf)
      const f4_t y = d[u][0], z = d[u][1];
      top[u] = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])));
      top[u] = fmaxf(top[u] * f[u], kNoScore);
    }
    const float change = unit.next(s_v);
    bool moved = false;
    if (__builtin_amdgcn_ballot_w64(top[0] - m[0] > kTop || top[1] - m[1] > kTop)) {
      // the rows' maxima over their four lanes; rows above the limit move their reference
      moved = true;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float t = fmaxf(top[u], __shfl_xor(top[u], 16));
        t = fmaxf(t, __shfl_xor(t, 32));
        const float mn = t - m[u] > kTop ? t + (kHeadroom - kTop) : m[u];
        alpha[u] = __builtin_amdgcn_exp2f(m[u] - mn);
        m[u] = mn;
        l[u] *= alpha[u];
      }
    }
    before();
    u4_t hw[2], lw[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float bias = unit.up - m[u];
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float x0 = d[u][t >> 1][2 * (t & 1)], x1 = d[u][t >> 1][2 * (t & 1) + 1];
        const float p0 = __builtin_amdgcn_exp2f(fmaf(x0, f[u], bias)), p1 = __builtin_amdgcn_exp2f(fmaf(x1, f[u], bias));
        sum += p0 + p1;
        const block_ops::Halves h = block_ops::split(p0, p1);
        hw[u][t] = h.hi;
        lw[u][t] = h.lo;
      }
      l[u] = fmaf(sum, unit.down, l[u]);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      ph[u] = __builtin_bit_cast(h8_t, hw[u]);
      pl[u] = __builtin_bit_cast(h8_t, lw[u]);
    }
    if (moved || change != 1.f) {  // after the products that belong to the old references
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int t = 0; t < 8; ++t) acc[u][t] *= alpha[u] * change;
    }
  };

  // packed blocks.  (LDS of the part before is read: its last barrier is behind that.)
  const int b0 = wk.b0, pe = min(wk.b1, rb.packed);
  if (b0 < pe) {
    Staged<NW> s0, s1;
    load(b0, s0);
    load(min(b0 + 1, pe - 1), s1);
#pragma unroll
    for (int u = 0; u < 2; ++u) ksc[u] = a.qscale * block_ops::lift_query(q[u]);
    for (int i = threadIdx.x; i < 8 * 64; i += 64 * NW)  // the values before the first block: zeros, of weights 0
      sm.op[(b0 - 1) & (kSlots - 1)][8 + (i >> 6)][i & 63] = (u4_t){0u, 0u, 0u, 0u};
    put(b0, s0);
    load(min(b0 + 2, pe - 1), s0);
    put(b0 + 1, s1);
    load(min(b0 + 3, pe - 1), s1);
    __syncthreads();
    f4_t d[2][2], next[2][2];
    scores(b0, d);
    // LDS holds b - 1 (values), b, b + 1; b + 2 is written, b + 4 asked for (past the last
    // block: that one again, unused)
    for (int b = b0; b < pe; ++b) {
      put(b + 2, s0);
      s0 = s1;
      load(min(b + 4, pe - 1), s1);
      const float2 sc = sm.scale[b & (kSlots - 1)];
      softmax(b, d, sc.x, block_ops::uniform(sc.y), [&]() { scores(b + 1, next); }, [&]() { values(b - 1); });
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int mb = 0; mb < 2; ++mb) d[u][mb] = next[u][mb];
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
    softmax(b, d, 1.f, 1.f, []() {}, []() {});
    tail_values(b);
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
      const float r = unit.ref / l[u];
      float* o = a.out + ((size_t)S.seq * a.nqry * a.hq + at[u]) * kHeadDim + 4 * blk;
#pragma unroll
      for (int t = 0; t < 8; ++t) *reinterpret_cast<f4_any*>(o + 16 * t) = acc[u][t] * r;
    } else {
      float* rec = a.ws + ((size_t)(S.ws_base + wk.split) * a.hq * a.nqry + at[u]) * kRecFloats;
#pragma unroll
      for (int t = 0; t < 8; ++t) *reinterpret_cast<f4_t*>(rec + 4 + 16 * t + 4 * blk) = acc[u][t] * unit.ref;
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
  __shared__ __attribute__((aligned(16))) Operands sm;
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
