// Pieces shared by the append kernels of the packed and the block-scaled caches:
// row loads, and the copy of the tokens that stay fp16 into the ring.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "kvq_internal.h"
#include "rotary.h"

namespace kvq {
namespace {

typedef uint32_t u4_t __attribute__((ext_vector_type(4)));

// 8 halves of a row at p: one 16-byte load, or halves (inputs that are not
// 16-byte aligned).
template <bool AL>
__device__ __forceinline__ u4_t load8(const uint16_t* p) {
  if constexpr (AL) return *reinterpret_cast<const u4_t*>(p);
  u4_t v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (uint32_t)p[2 * i] | ((uint32_t)p[2 * i + 1] << 16);
  return v;
}
template <bool AL>
__device__ __forceinline__ uint32_t load2(const uint16_t* p) {
  if constexpr (AL) return *reinterpret_cast<const uint32_t*>(p);
  return (uint32_t)p[0] | ((uint32_t)p[1] << 16);
}

// Row of token p: in the ring (appended by an earlier call) or in the input.
struct Rows {
  const uint16_t* in;    // input row of token L_old of this head
  const uint16_t* ring;
  size_t stride;         // halves from one input token to the next
  int L_old, W;
  bool fresh;            // none of the group's tokens sits in the ring (uniform)
  __device__ __forceinline__ const uint16_t* at(int p) const {
    if (!fresh && p < L_old) return ring + (size_t)(p % W) * kHeadDim;
    return in + (size_t)(p - L_old) * stride;
  }
};

// The sequence of a workgroup: the last one that begins at it or before.  One load for
// all of them: asked for one after another, 64 of them took 15 us.
__device__ __forceinline__ int sequence_of(const AppendArgs& a, int wg) {
  static_assert(kMaxSeqPerLaunch <= 64, "one lane per sequence");
  if (a.nseq == 1) return 0;
  const int lane = threadIdx.x & 63;
  const auto* args = (const AppendArgs*)__builtin_amdgcn_kernarg_segment_ptr();  // (indexed by lane, `a` would be copied)
  const int begin = args->seq[min(lane, kMaxSeqPerLaunch - 1)].wg_begin;
  return __popcll(__builtin_amdgcn_ballot_w64(lane < a.nseq && begin <= wg)) - 1;
}

// Workgroup `local` of parts x hkv as (part, kv head).  The heads of a part sit 8 apart,
// on one XCD, whose L2 then holds its tokens' angles for all of them.
struct PartHead {
  int part, h;
};
__device__ __forceinline__ PartHead part_head(int local, int parts, int hkv) {
  const int chunk = local / (8 * hkv), r = local - chunk * 8 * hkv;
  if (8 * chunk + 8 <= parts) return {8 * chunk + (r & 7), r >> 3};
  return {8 * chunk + r / hkv, r % hkv};
}

// Copy part `part` (kCopyTokens tokens) of the new tokens that stay fp16 into
// the ring of head h.  Turned keys and converted values may have left fp16's range:
// attention reads them before their group is packed, so they are reported here.
template <bool AL, int ROT>
__device__ __forceinline__ void copy_ring(const AppendArgs& a, const RotaryArgs* rot, const AppendSeq& S, int h, int part) {
  uint8_t* blk = a.arena + S.head0 + (uint64_t)h * a.head_stride;
  const int first = max(S.Lq_new, S.L_old) + part * kCopyTokens, end = min(S.L_new, first + kCopyTokens);
  const size_t token0 = (size_t)S.seq * a.n_max, ks = ROT ? rot->k_stride : (size_t)a.hkv * kHeadDim,
               vs = ROT ? rot->v_stride : (size_t)a.hkv * kHeadDim;
  constexpr int kPer = kCopyTokens * (kHeadDim / 8) / kAppendThreads;  // 16-byte pieces per thread and tensor
  u4_t x[2][kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int idx = i * kAppendThreads + threadIdx.x, p = first + (idx >> 4);
    if (p < end) {
      const size_t token = token0 + (p - S.L_old), at = (size_t)h * kHeadDim + (idx & 15) * 8;
      x[0][i] = load8<AL>(a.K + token * ks + at);
      x[1][i] = load8<AL>(a.V + token * vs + at);
      if constexpr (ROT) {
        const rotary::Turn<ROT> turn(*rot, threadIdx.x & 63);
        rotary::Angles g;
        turn.load(*rot, rotary::table_row(*rot, a.arena, (int64_t)token, p), g);
        x[0][i] = turn.apply(x[0][i], g);
#pragma unroll
        for (int n = 0; n < 4; ++n) x[1][i][n] = rotary::to_half2<ROT>(x[1][i][n]);
        rotary::report_range(a.arena, x[0][i], x[1][i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int idx = i * kAppendThreads + threadIdx.x, p = first + (idx >> 4);
    if (p < end) {
      const size_t dst = ((size_t)(p % a.W) * kHeadDim + (idx & 15) * 8) * 2;
      *reinterpret_cast<u4_t*>(blk + region(a.tk) + dst) = x[0][i];
      *reinterpret_cast<u4_t*>(blk + region(a.tv) + dst) = x[1][i];
    }
  }
}

}  // namespace
}  // namespace kvq
