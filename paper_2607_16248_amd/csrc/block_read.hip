// Reading a block-scaled cache back (gfx950): dequantized values of a token range
// (kvq_dequant) and the canonical image of a head (kvq_export).  One workgroup takes
// a 32-token block of a head; the values' codes, which lie in operand order, turn
// through LDS.  Bound by the writes: 16384 tokens and 8 kv heads, keys
// and values as fp32 and their codes, 168 MB, 34 us (4.9 TB/s).
#include <hip/hip_runtime.h>

#include "kvq_internal.h"
#include "kvq_layout.h"

namespace kvq {
namespace {

constexpr int kThreads = 256;
typedef float f4_t __attribute__((ext_vector_type(4)));
typedef f4_t f4_any __attribute__((aligned(4)));

// Two bytes of w (the lower, or with hi the upper ones) as numbers.
__device__ __forceinline__ void numbers4(uint32_t w, int type, float (&v)[4]) {
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const uint32_t b = (w >> (8 * n)) & 0xFFu;
    v[n] = (float)((int)b - 128);
  }
  if (type != kBlockE4M3) return;
  typedef float f2_t __attribute__((ext_vector_type(2)));
  const f2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  v[0] = lo.x;
  v[1] = lo.y;
  v[2] = hi.x;
  v[3] = hi.y;
}

// The 32 tokens of a block of value codes, row by row.
struct ValueTile {
  uint32_t w[1024];
  __device__ __forceinline__ void load(const uint8_t* p) {
    *reinterpret_cast<uint4*>(&w[4 * threadIdx.x]) = *reinterpret_cast<const uint4*>(p + 16 * threadIdx.x);
  }
  // channels c .. c + 3 (c a multiple of 4) of token r
  __device__ __forceinline__ uint32_t row4(int r, int c) const {
    const uint8_t* b = reinterpret_cast<const uint8_t*>(w);
    uint32_t v = 0u;
#pragma unroll
    for (int n = 0; n < 4; ++n) v |= (uint32_t)b[block_value(r, c + n)] << (8 * n);
    return v;
  }
};

__global__ __launch_bounds__(kThreads) void dequant_block_kernel(DequantArgs a) {
  __shared__ ValueTile tile;
  const int bi = blockIdx.x / a.hkv, h = blockIdx.x - bi * a.hkv;
  const int p0 = (a.tok0 & ~31) + 32 * bi, tid = threadIdx.x;
  const uint8_t* ring = a.arena + a.head0 + (uint64_t)h * a.head_stride;
  const bool packed = p0 < a.Lq;  // (Lq is a multiple of 32: a block is packed or not)
  const uint8_t* kc = nullptr;
  float sk = 0.f, sv = 0.f;
  if (packed) {
    int t0;
    const uint8_t* seg = a.arena + packed_seg(a.pm, a.head0, a.head_stride, a.seq, h, p0, t0);
    kc = seg + region(a.kc) + (size_t)t0 * kHeadDim;
    const float* sc = reinterpret_cast<const float*>(seg + region(a.km)) + (size_t)(t0 / a.gk) * 2;
    sk = sc[0];
    sv = sc[1];
    tile.load(seg + region(a.vc) + (size_t)t0 * kHeadDim);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int idx = i * kThreads + tid, r = idx >> 5, c = 4 * (idx & 31), p = p0 + r;
    if (p < a.tok0 || p >= a.tok0 + a.ntok) continue;
    const size_t o = ((size_t)(p - a.tok0) * a.hkv + h) * kHeadDim + c;
    float k[4], v[4];
    if (packed) {
      numbers4(*reinterpret_cast<const uint32_t*>(kc + r * kHeadDim + c), a.bk, k);
      numbers4(tile.row4(r, c), a.bv, v);
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        k[n] *= sk;
        v[n] *= sv;
      }
    } else {
      typedef _Float16 h4_t __attribute__((ext_vector_type(4)));
      const size_t at = (size_t)(p % a.W) * kHeadDim + c;
      const h4_t x = *reinterpret_cast<const h4_t*>(reinterpret_cast<const _Float16*>(ring + region(a.tk)) + at);
      const h4_t y = *reinterpret_cast<const h4_t*>(reinterpret_cast<const _Float16*>(ring + region(a.tv)) + at);
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        k[n] = (float)x[n];
        v[n] = (float)y[n];
      }
    }
    *reinterpret_cast<f4_any*>(a.K_out + o) = (f4_t){k[0], k[1], k[2], k[3]};
    *reinterpret_cast<f4_any*>(a.V_out + o) = (f4_t){v[0], v[1], v[2], v[3]};
  }
}

__device__ __forceinline__ void put4(uint8_t* p, uint32_t v) {  // (an image begins anywhere)
#pragma unroll
  for (int n = 0; n < 4; ++n) p[n] = (uint8_t)(v >> (8 * n));
}

__global__ __launch_bounds__(kThreads) void export_block_kernel(ExportArgs a) {
  __shared__ ValueTile tile;
  const int p0 = 32 * blockIdx.x, tid = threadIdx.x;
  if (p0 < a.Lq) {
    int t0;
    const uint8_t* seg = a.arena + packed_seg(a.pm, a.head0, a.head_stride, a.seq, a.h, p0, t0);
    tile.load(seg + region(a.vc) + (size_t)t0 * kHeadDim);
    __syncthreads();
    const uint32_t fk = a.bk == kBlockE4M3 ? 0u : 0x80808080u, fv = a.bv == kBlockE4M3 ? 0u : 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int idx = i * kThreads + tid, r = idx >> 5, c = 4 * (idx & 31);
      const uint32_t k = *reinterpret_cast<const uint32_t*>(seg + region(a.kc) + (size_t)(t0 + r) * kHeadDim + c);
      put4(a.kc_out + (size_t)(p0 + r) * kHeadDim + c, k ^ fk);
      put4(a.vc_out + (size_t)(p0 + r) * kHeadDim + c, tile.row4(r, c) ^ fv);
    }
    if (p0 % a.gk == 0 && tid < 2) {
      const uint32_t s = reinterpret_cast<const uint32_t*>(seg + region(a.km))[(size_t)(t0 / a.gk) * 2 + tid];
      put4((tid ? a.vm_out : a.km_out) + (size_t)(p0 / a.gk) * 4, s);
    }
    return;
  }
  const uint8_t* ring = a.arena + a.head0 + (uint64_t)a.h * a.head_stride;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int idx = i * kThreads + tid, r = idx >> 6, c = 4 * (idx & 63), p = p0 + r;  // c: byte of the row
    if (p >= a.Lq + a.ntail) continue;
    const size_t at = (size_t)(p % a.W) * kHeadDim * 2 + c, o = (size_t)(p - a.Lq) * kHeadDim * 2 + c;
    put4(a.tk_out + o, *reinterpret_cast<const uint32_t*>(ring + region(a.tk) + at));
    put4(a.tv_out + o, *reinterpret_cast<const uint32_t*>(ring + region(a.tv) + at));
  }
}

}  // namespace

int launch_dequant_block(const DequantArgs& a, void* stream) {
  const int64_t blocks = ((int64_t)a.tok0 + a.ntok + 31) / 32 - a.tok0 / 32;
  hipLaunchKernelGGL(dequant_block_kernel, dim3((unsigned)(blocks * a.hkv)), dim3(kThreads), 0, (hipStream_t)stream, a);
  return (int)hipGetLastError();
}

int launch_export_block(const ExportArgs& a, void* stream) {
  const int64_t blocks = ((int64_t)a.Lq + a.ntail + 31) / 32;
  hipLaunchKernelGGL(export_block_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a);
  return (int)hipGetLastError();
}

}  // namespace kvq
