// Attention of few rows over a block-scaled cache (gfx950; include/kvq.h states
// both): single-token decode, chunk queries and windows, up to 16 or 32 (query, head)
// rows of a kv head.
//
//   S^T = K Q^T   (16 tokens x 16 rows; codes as exact halves, q as the fp16 it is)
//   p = 2^(s_k c S + log2 s_v - m),   O^T += V^T P^T   (p in hi + lo halves)
//
// with s_k, s_v the block's scales: one number each for all 32 tokens that a wave
// takes at a time, so they enter as factors of scores and weights, and codes stay
// the integers (or e4m3 numbers) they are.  The reference m of a row goes by what its
// weights contribute, not by the scores alone: values of blocks far apart in size keep
// their bits.  Products are transposed, so a lane's
// weights are the next product's operand without a lane exchange.  A lane reads 16
// consecutive bytes of a key row (any order of channels does, the query has the
// same), and values lie in operand order (kvq_layout.h, block_value).
//
// A workgroup's four waves take 32-token blocks in turn; the next block's codes are
// asked for before this one's are used.  Work is split by its amount: the key groups
// of all sequences and kv heads are one list, of which every workgroup takes the same
// number, whatever heads they belong to (sequences of different lengths would
// otherwise leave compute units idle).  The part that holds a head's end adds the
// fp16 tail (tail_mfma.h); a sequence whose heads are whole in their workgroups is
// written to the output, else its parts are joined by the merge launch.
//
// Single tokens are bound by memory: 32 sequences of 9000 to 16384 tokens, 8 kv heads,
// 847 MB of e4m3, 143 us (5.9 TB/s; a reading probe reaches 6.4).  With 32 rows (five
// queries of four heads over 4 sequences of 20000 to 32768 tokens, 222 MB) it is the
// latency of a wave's block, whose products and weights follow one another, and the
// registers: two tiles take all 256 and spill 62 (252 bytes of scratch a lane; one tile
// takes 207 to 209 and spills none): 75 us (3.0 TB/s).  Over 4 sequences of 32768 one query
// takes 50 us, four (one tile) 59, five (two) 70.  Two blocks of a wave in turn need more.
#include <hip/hip_runtime.h>

#include "block_ops.h"
#include "decode_common.h"
#include "kvq_internal.h"
#include "kvq_layout.h"
#include "mfma_common.h"
#include "tail_mfma.h"

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

// What a wave reads of a 32-token block.
struct Codes {
  u4_t k[4];  // token half, 64-channel half
  u4_t v[4];  // pieces
};

// The waves' results of a part, joined through LDS.
template <int NT>
struct Joined {
  float m[kWaves][16 * NT], l[kWaves][16 * NT];
  float acc[kWaves][16 * NT][kHeadDim + 4];  // (rows begin in distinct banks)
};

// Codes that one workgroup reads once (ONCE: past the caches, 188 us to 168 at 32
// sequences of 9000 to 16384 tokens), or several row groups.
template <bool ONCE>
__device__ __forceinline__ u4_t load_codes(const uint8_t* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const u4_t*>(p));
  return *reinterpret_cast<const u4_t*>(p);
}

// The part [u0, u1) of the units of one (sequence, kv head, row group): its key groups
// and, as the last unit that stands for work, the fp16 tail.
struct Part {
  int si, h, rg, u0, u1, split;
};

// NT: tiles of 16 rows.
template <bool K8, bool V8, int NT, bool ONCE>
__device__ __forceinline__ void attend_part(const DecodeArgs& a, const Part& wk, Joined<NT>& red) {
  const DecodeSeq& S = a.seq[wk.si];
  const uint8_t* ring = a.arena + S.head0 + (uint64_t)wk.h * a.head_stride;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, blk = lane >> 4;
  const int rows = a.qpr * a.gqh;  // of the group
  const int inv = (65536 + a.gqh - 1) / a.gqh;
  const size_t rec_rows = (size_t)a.hq * a.nqry;

  const int seen0 = S.L - a.nqry + 1;
  const int first_limit = seen0 + min(wk.rg * a.qpr, a.nqry - 1);
  const int last_limit = seen0 + min(wk.rg * a.qpr + a.qpr - 1, a.nqry - 1);
  const int gsh = __builtin_ctz(a.gk), bsh = gsh - 5;
  const WindowGroups wg = window_groups(first_limit, last_limit, S.Lq, gsh, a.window, a.sinks);
  // 32-token blocks of this part, every fourth one this wave's
  const int i0 = (wk.u0 << bsh) + wv, iend = min(wg.count, wk.u1) << bsh;
  const int nblocks = i0 < iend ? (iend - i0 + kWaves - 1) / kWaves : 0;
  auto token_of = [&](int i) {
    i = i0 + kWaves * i;
    const int j = i >> bsh;
    return (i << 5) + (j < wg.sink ? 0 : (wg.first - wg.sink) << gsh);
  };

  // The page of a block's tokens and its scales come by vector loads, whose results
  // arrive in the order asked for: pages two blocks ahead, scales ahead of the keys.
  // (Scalar loads, which are waited for all at once, took as long.)
  const bool paged = a.pm.table != nullptr;
  const uint8_t* head = a.arena + (paged ? a.pm.pool0 + (uint64_t)wk.h * a.pm.page_head_bytes : S.head0 + (uint64_t)wk.h * a.head_stride);
  const int32_t* table = a.pm.table + (size_t)S.seq * a.pm.max_pages;
  const int page_shift = paged ? a.pm.page_shift : 31, in_page = paged ? a.pm.page_tokens - 1 : 0x7FFFFFFF;
  const uint64_t page_bytes = paged ? a.pm.page_bytes : 0;
  int zero = 0;
  asm("" : "+v"(zero));  // (keeps the loads' addresses in vector registers)
  auto page_of = [&](int i) { return paged ? table[(token_of(i) >> page_shift) + zero] : 0; };
  const uint32_t k_at = col * kHeadDim + 16 * blk, v_at = lane * 16;
  // rows 16 u + col of the group: query operands and limits (rows past whole
  // queries, and queries past the last, repeat the last query)
  u4_t q[NT][4];
  int lim[NT];
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    typedef u4_t u4_any __attribute__((aligned(4)));
    const int g = 16 * u + col, x = (g * inv) >> 16, j = min(wk.rg * a.qpr + (x < a.qpr ? x : kSpareRow), a.nqry - 1);
    lim[u] = seen0 + j;
    const uint16_t* qr = a.q + (((size_t)S.seq * a.nqry + j) * a.hq + wk.h * a.gqh + (g - x * a.gqh)) * kHeadDim + 16 * blk;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) q[u][kb] = *reinterpret_cast<const u4_any*>(qr + 64 * (kb >> 1) + 8 * (kb & 1));
  }
  Codes code;
  auto segment = [&](int i, int page, int& t) {
    t = token_of(i) & in_page;
    return head + (uint64_t)(uint32_t)page * page_bytes;
  };
  auto load_keys = [&](int i, int page) __attribute__((always_inline)) {
    int t;
    const uint8_t* seg = segment(i, page, t);
    const uint8_t* kr = seg + region(a.kc) + (size_t)t * kHeadDim;
#pragma unroll
    for (int n = 0; n < 4; ++n) code.k[n] = load_codes<ONCE>(kr + (n >> 1) * 16 * kHeadDim + (n & 1) * 64 + k_at);
  };
  auto load_values = [&](int i, int page) __attribute__((always_inline)) {
    int t;
    const uint8_t* seg = segment(i, page, t);
    const uint8_t* vr = seg + region(a.vc) + (size_t)t * kHeadDim;
#pragma unroll
    for (int n = 0; n < 4; ++n) code.v[n] = load_codes<ONCE>(vr + n * 1024 + v_at);
  };
  float2 scale = make_float2(0.f, 0.f);
  auto load_scales = [&](int i, int page) __attribute__((always_inline)) {
    int t;
    const uint8_t* seg = segment(i, page, t);
    scale = *reinterpret_cast<const float2*>(seg + region(a.km) + (size_t)((t >> gsh) + zero) * 8);
  };
  const int last = nblocks - 1;
  int page = 0;
  if (nblocks > 0) {  // under way while the queries are waited for
    const int first = __builtin_amdgcn_readfirstlane(page_of(0));
    page = page_of(min(1, last));
    load_scales(0, first);
    load_keys(0, first);
    load_values(0, first);
  }

  float ksc[NT];
#pragma unroll
  for (int u = 0; u < NT; ++u) ksc[u] = a.qscale * block_ops::lift_query(q[u]);
  float m[NT], l[NT];
  f4_t acc[NT][8];
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    m[u] = kNoScore;
    l[u] = 0.f;
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[u][t] = (f4_t){0.f, 0.f, 0.f, 0.f};
  }

  // block i; the next one's keys are asked for when this one has its scores, its
  // values and scales when this one is done
  auto attend = [&](int i) __attribute__((always_inline)) {
    const int next = min(i + 1, last);  // (after the last block: that one again, unused)
    const float s_k = block_ops::uniform(scale.x), s_v = block_ops::uniform(scale.y);
    const float up = block_ops::log_scale(s_v), down = __builtin_amdgcn_exp2f(-up);
    f4_t d[NT][2];
#pragma unroll
    for (int mb = 0; mb < 2; ++mb) {
#pragma unroll
      for (int u = 0; u < NT; ++u) d[u][mb] = (f4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        const u4_t w = code.k[2 * mb + (kb >> 1)];
        const h8_t k8 = block_ops::operand<K8>(w[2 * (kb & 1)], w[2 * (kb & 1) + 1]);
#pragma unroll
        for (int u = 0; u < NT; ++u) d[u][mb] = mfma(k8, __builtin_bit_cast(h8_t, q[u][kb]), d[u][mb]);
      }
    }
    const int at = __builtin_amdgcn_readfirstlane(page);
    page = page_of(min(i + 2, last));
    load_scales(next, at);
    load_keys(next, at);
    const int tok = token_of(i);
    if (tok + 32 > first_limit || (tok < last_limit - a.window && tok + 32 > a.sinks)) {
      // token tok + 16mb + 4blk + r is visible below the limit, from the window's
      // begin on or below the sinks' end
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        const int left = lim[u] - tok - 4 * blk, from = max(lim[u] - a.window, 0) - tok - 4 * blk, sunk = a.sinks - tok - 4 * blk;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int n = 16 * (e >> 2) + (e & 3);
          float s = n < left && (n >= from || n < sunk) ? d[u][e >> 2][e & 3] : -__builtin_inff();
          asm volatile("" : "+v"(s));  // (a branch: blocks within every window pass it by)
          d[u][e >> 2][e & 3] = s;
        }
      }
    }
    h8_t ph[NT], pl[NT];
    float top[NT], f[NT];
    bool over = false;
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      f[u] = ksc[u] * (s_k > 0.f ? s_k : 1.f);  // (a block of zeros has scores 0 at any scale; a hidden token's is -inf)
      const f4_t y = d[u][0], z = d[u][1];
      top[u] = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])));
      top[u] = fmaxf(fmaf(top[u], f[u], up), kNoScore);
      over |= top[u] - m[u] > kTop;
    }
    if (__builtin_amdgcn_ballot_w64(over)) {
      // the rows' maxima over their four lanes; rows above the limit move their reference
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        float t = fmaxf(top[u], __shfl_xor(top[u], 16));
        t = fmaxf(t, __shfl_xor(t, 32));
        const float mn = t - m[u] > kTop ? t + (kHeadroom - kTop) : m[u];
        const float alpha = __builtin_amdgcn_exp2f(m[u] - mn);
        m[u] = mn;
        l[u] *= alpha;
#pragma unroll
        for (int t2 = 0; t2 < 8; ++t2) acc[u][t2] *= alpha;
      }
    }
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      const float bias = up - m[u];
      float sum = 0.f;
      u4_t hw, lw;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float s0 = d[u][t >> 1][2 * (t & 1)], s1 = d[u][t >> 1][2 * (t & 1) + 1];
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s0, f[u], bias)), p1 = __builtin_amdgcn_exp2f(fmaf(s1, f[u], bias));
        sum += p0 + p1;
        const block_ops::Halves h = block_ops::split(p0, p1);
        hw[t] = h.hi;
        lw[t] = h.lo;
      }
      l[u] = fmaf(sum, down, l[u]);
      ph[u] = __builtin_bit_cast(h8_t, hw);
      pl[u] = __builtin_bit_cast(h8_t, lw);
    }
#pragma unroll
    for (int mb = 0; mb < 8; ++mb) {
      const u4_t w = code.v[mb >> 1];
      const h8_t v8 = block_ops::operand<V8>(w[2 * (mb & 1)], w[2 * (mb & 1) + 1]);
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        acc[u][mb] = mfma(v8, ph[u], acc[u][mb]);
        acc[u][mb] = mfma(v8, pl[u], acc[u][mb]);
      }
    }
    load_values(next, at);
  };

  for (int i = 0; i < nblocks; ++i) attend(i);

  TailState<NT> st;
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    l[u] += __shfl_xor(l[u], 16);
    l[u] += __shfl_xor(l[u], 32);
    st.m[u] = l[u] > 0.f ? m[u] : -__builtin_inff();
    st.l[u] = l[u];
#pragma unroll
    for (int t = 0; t < 8; ++t) st.acc[u][t] = acc[u][t];
  }
  if (S.L > S.Lq && wk.u1 == S.L_old) {  // the fp16 tail
    TailState<NT> tail;
    tail_split<NT, 16 * NT, true, 4, true>(a, S, wk.h, wk.rg, ring, tail, lane, wv);
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      const float top = fmaxf(st.m[u], tail.m[u]);  // (-inf in a wave that read nothing)
      const float f = st.l[u] > 0.f ? __builtin_amdgcn_exp2f(st.m[u] - top) : 0.f;
      const float ft = tail.l[u] > 0.f ? __builtin_amdgcn_exp2f(tail.m[u] - top) : 0.f;
      st.m[u] = top;
      st.l[u] = st.l[u] * f + tail.l[u] * ft;
#pragma unroll
      for (int t = 0; t < 8; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) st.acc[u][t][r] = st.acc[u][t][r] * f + tail.acc[u][t][r] * ft;
    }
  }

  __syncthreads();  // (the part before is read)
#pragma unroll
  for (int u = 0; u < NT; ++u) {
#pragma unroll
    for (int t = 0; t < 8; ++t) *reinterpret_cast<f4_t*>(&red.acc[wv][16 * u + col][16 * t + 4 * blk]) = st.acc[u][t];
    if (blk == 0) {
      red.m[wv][16 * u + col] = st.m[u];
      red.l[wv][16 * u + col] = st.l[u];
    }
  }
  __syncthreads();
  // a thread joins four channels of a row: into the output of a sequence of one part
  // (every row sees a token in it), else into a record
  for (int idx = threadIdx.x; idx < rows * (kHeadDim / 4); idx += blockDim.x) {
    const int g = idx / (kHeadDim / 4), c = 4 * (idx % (kHeadDim / 4)), x = (g * inv) >> 16, j = wk.rg * a.qpr + x;
    if (j >= a.nqry) continue;
    float M = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, red.m[w][g]);
    f4_t val = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = red.m[w][g] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(red.m[w][g] - M);
      const f4_t v = *reinterpret_cast<const f4_t*>(&red.acc[w][g][c]);
#pragma unroll
      for (int n = 0; n < 4; ++n) val[n] = fmaf(f, v[n], val[n]);
      sum = fmaf(f, red.l[w][g], sum);
    }
    const size_t row = (size_t)j * a.hq + wk.h * a.gqh + g - x * a.gqh;
    if (S.nsplit == 1) {
      typedef f4_t f4_any __attribute__((aligned(4)));
      *reinterpret_cast<f4_any*>(a.out + ((size_t)S.seq * rec_rows + row) * kHeadDim + c) = val / (f4_t){sum, sum, sum, sum};
    } else {
      float* rec = a.ws + ((size_t)(S.ws_base + wk.split) * rec_rows + row) * kRecFloats;
      *reinterpret_cast<f4_t*>(rec + 4 + c) = val;
      if (c == 0) { rec[0] = M; rec[1] = sum; }
    }
  }
  // row groups of one sequence have one number of records: those of fewer parts end
  // with empty ones
  if (wk.u1 == S.L_old) {
    for (int split = wk.split + 1; split < S.nsplit; ++split)
      for (int idx = threadIdx.x; idx < rows * kRecFloats; idx += blockDim.x) {
        const int g = idx / kRecFloats, c = idx - g * kRecFloats, x = (g * inv) >> 16, j = wk.rg * a.qpr + x;
        if (j >= a.nqry) continue;
        const size_t row = (size_t)j * a.hq + wk.h * a.gqh + g - x * a.gqh;
        a.ws[((size_t)(S.ws_base + split) * rec_rows + row) * kRecFloats + c] = c == 0 ? -__builtin_inff() : 0.f;
      }
  }
}

// The units of a launch (a key group each, and those that stand for a tail) lie one
// (sequence, kv head, row group) after the other; a workgroup takes
// a.units_per_wg of them, whatever they belong to.
template <bool K8, bool V8, int NT, bool ONCE>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void block_tiles_kernel(DecodeArgs a) {
  __shared__ __attribute__((aligned(16))) Joined<NT> red;
  const int per = a.units_per_wg, end = min((int)(blockIdx.x + 1) * per, a.total_wg);
  for (int u = blockIdx.x * per; u < end;) {
    Part p;
    p.si = block_ops::sequence_of(a, u);
    const DecodeSeq& S = a.seq[p.si];
    const int at = u - S.wg_begin, seg = at / S.nq, begin = S.wg_begin + seg * S.nq;
    p.h = seg / a.nrg;
    p.rg = seg - p.h * a.nrg;
    p.u0 = u - begin;
    p.u1 = min(S.L_old, end - begin);
    p.split = (int)blockIdx.x - begin / per;
    if (p.u0 < p.u1) attend_part<K8, V8, NT, ONCE>(a, p, red);
    u = begin + S.nq;
  }
}

template <bool K8, bool V8>
int launch_types(const DecodeArgs& a, int rows, void* stream) {
  const dim3 grid((unsigned)((a.total_wg + a.units_per_wg - 1) / a.units_per_wg)), block(64 * kWaves);
  hipStream_t s = (hipStream_t)stream;
  if (a.nrg > 1) {
    if (rows > 16) hipLaunchKernelGGL((block_tiles_kernel<K8, V8, 2, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((block_tiles_kernel<K8, V8, 1, false>), grid, block, 0, s, a);
  } else {
    if (rows > 16) hipLaunchKernelGGL((block_tiles_kernel<K8, V8, 2, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((block_tiles_kernel<K8, V8, 1, true>), grid, block, 0, s, a);
  }
  return (int)hipGetLastError();
}

}  // namespace

int launch_block_tiles(const DecodeArgs& a, int type_k, int type_v, int rows, void* stream) {
  if (a.total_wg <= 0) return 0;
  if (type_k == kBlockE4M3)
    return type_v == kBlockE4M3 ? launch_types<true, true>(a, rows, stream) : launch_types<true, false>(a, rows, stream);
  return type_v == kBlockE4M3 ? launch_types<false, true>(a, rows, stream) : launch_types<false, false>(a, rows, stream);
}

}  // namespace kvq
