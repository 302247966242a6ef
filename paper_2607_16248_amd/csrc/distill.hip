// The loss of a student's logits against a teacher's top logits, and its
// gradient (gfx950; include/dgap.h states both).
//
//   loss_r = T^2 sum_k q_k (log q_k - log p_{i_k}),  p = softmax(z / T) over the
//   vocabulary, q = softmax(t / T) over the row's entries;
//   d loss_r / d z_j = T (p_j - sum_k q_k [i_k = j]).
//
// Bound by memory: the loss reads every logit once, the gradient reads and
// writes each once more.  Exponentials in base 2 with c = log2(e) / T in two
// parts, so that an argument z c - m is off by no more than its own rounding.
//   sums   one workgroup per (row, chunk): the chunk's maximum and its sum
//   loss   one wave per row: the chunks joined, the entries' q, the loss
//   grad   one workgroup per (row, chunk): q goes to the chunk's places in LDS
//          (entries of one index added in their order), then the logits pass
//          through: every thread writes the gradient of what it read, so the
//          gradient may take the logits' place
#include <hip/hip_runtime.h>

#include "decode_common.h"
#include "kvq_internal.h"
#include "logits_common.h"

namespace kvq {
namespace {

using namespace logits;

constexpr int kThreads = 256;
constexpr int kPer = kDistillChunk / kThreads;  // logits per thread, in runs of 8
constexpr int kMaxK = kDistillMaxK;

// 8 consecutive logits; those from `n` on read as -inf
template <class T>
__device__ __forceinline__ void load_part(const typename T::raw* p, int n, float (&v)[8]) {
  raw8_t<T> x = all8<T>(-__builtin_inff());
  if (n >= 8) {
    x = load8<T>(p);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) x[j] = p[j];
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = T::value(x[j]);
}

// T's gradient or loss entry of a row: its place, its share q (0: no entry)
struct Entry {
  int index;
  float q;
};

// 2^(x c - less): x, a difference to the largest logit, is taken before c, so
// that neither the type's lowest value nor a whole row of it overflows
__device__ __forceinline__ float power(float x, const DistillArgs& a, float less) {
  return __builtin_amdgcn_exp2f(fmaf(x, a.c, fmaf(x, a.c_low, -less)));
}

template <class T>
__global__ __launch_bounds__(kThreads) void distill_sums_kernel(DistillArgs a) {
  __shared__ float wm[kThreads / 64], ws[kThreads / 64];
  const int row = blockIdx.x / a.nchunk, chunk = blockIdx.x % a.nchunk, tid = threadIdx.x;
  const auto* z = reinterpret_cast<const typename T::raw*>(a.logits) + (size_t)row * a.row_stride;
  const int from = chunk * kDistillChunk;
  float v[kPer / 8][8], m = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < kPer / 8; ++i) {
    const int at = from + 8 * (i * kThreads + tid);
    load_part<T>(z + at, a.vocab - at, v[i]);
  }
#pragma unroll
  for (int i = 0; i < kPer / 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, v[i][j]);
  m = dec::wave_max(m);
  if ((tid & 63) == 0) wm[tid >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) m = fmaxf(m, wm[w]);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kPer / 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) s += v[i][j] == -__builtin_inff() ? 0.f : power(v[i][j] - m, a, 0.f);
  s = dec::wave_sum(s);
  if ((tid & 63) == 0) ws[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) {
    float* o = a.ws + ((size_t)row * a.nchunk + chunk) * 2;
    o[0] = m;
    o[1] = (ws[0] + ws[1]) + (ws[2] + ws[3]);
  }
}

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// The row's entries, up to kMaxK / 64 per lane of a wave: places and base-2
// logits t c - max (0 weight where there is no entry).
struct Entries {
  int index[kMaxK / 64];
  double x[kMaxK / 64], w[kMaxK / 64], total;
  bool any;
};
__device__ __forceinline__ Entries entries_of(const DistillArgs& a, int row, int lane) {
  Entries e;
  float t[kMaxK / 64], top = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < kMaxK / 64; ++i) {
    const int k = 64 * i + lane;
    e.index[i] = k < a.k ? a.index[(size_t)row * a.k + k] : -1;
    t[i] = k < a.k ? a.teacher[(size_t)row * a.k + k] : -__builtin_inff();
    if ((uint32_t)e.index[i] >= (uint32_t)a.vocab || t[i] == -__builtin_inff()) e.index[i] = -1;
    if (e.index[i] >= 0) top = fmaxf(top, t[i]);
  }
  top = dec::wave_max(top);
  e.any = top != -__builtin_inff();
  const double c = (double)a.c + (double)a.c_low;
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < kMaxK / 64; ++i) {
    e.x[i] = ((double)t[i] - (double)top) * c;
    e.w[i] = e.index[i] >= 0 ? exp2(e.x[i]) : 0.0;
    sum += e.w[i];
  }
  e.total = wave_sum_d(sum);
  return e;
}

template <class T>
__global__ __launch_bounds__(kThreads) void distill_loss_kernel(DistillArgs a) {
  const int row = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= a.rows) return;
  const auto* z = reinterpret_cast<const typename T::raw*>(a.logits) + (size_t)row * a.row_stride;
  const float* part = a.ws + (size_t)row * a.nchunk * 2;
  const double c = (double)a.c + (double)a.c_low;
  float m = -__builtin_inff();
  for (int i = lane; i < a.nchunk; i += 64) m = fmaxf(m, part[2 * i]);
  m = dec::wave_max(m);
  double s = 0.0;
  for (int i = lane; i < a.nchunk; i += 64)
    if (part[2 * i + 1] != 0.f) s += (double)part[2 * i + 1] * exp2(((double)part[2 * i] - (double)m) * c);
  const double log_sum = log2(wave_sum_d(s));  // of 2^((z - m) c)
  const Entries e = entries_of(a, row, lane);
  const double log_total = e.any ? log2(e.total) : 0.0;
  double loss = 0.0;
#pragma unroll
  for (int i = 0; i < kMaxK / 64; ++i)
    if (e.index[i] >= 0)
      loss += e.w[i] / e.total * (e.x[i] - log_total - ((double)T::value(z[e.index[i]]) - (double)m) * c + log_sum);
  loss = wave_sum_d(loss);
  if (lane == 0) {
    a.loss[row] = (float)(loss * 0.6931471805599453 * (double)a.temperature * (double)a.temperature);
    if (a.lse) a.lse[row] = (float)((log_sum + (double)m * c) * 0.6931471805599453);
    if (a.grad) {  // for the gradient's launch
      a.row_sum[2 * row] = m;
      a.row_sum[2 * row + 1] = (float)log_sum;
    }
  }
}

// 8 values to p, which has its element's alignment only
template <class T>
__device__ __forceinline__ void store8(typename T::raw* p, int n, const float (&v)[8]) {
  typedef typename T::raw vec __attribute__((ext_vector_type(8)));
  typedef vec vec_any __attribute__((aligned(sizeof(typename T::raw))));
  if (n >= 8) {
    vec x;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = T::make(v[j]);
    *reinterpret_cast<vec_any*>(p) = x;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = T::make(v[j]);
  }
}

// OWN_SUM: with what distill_loss_kernel left, else from the caller's lse
template <class T, bool OWN_SUM>
__global__ __launch_bounds__(kThreads) void distill_grad_kernel(DistillArgs a) {
  __shared__ __attribute__((aligned(16))) float share[kDistillChunk];
  __shared__ Entry entry[kMaxK];
  __shared__ int some;
  const int row = blockIdx.x / a.nchunk, chunk = blockIdx.x % a.nchunk, tid = threadIdx.x;
  const auto* z = reinterpret_cast<const typename T::raw*>(a.logits) + (size_t)row * a.row_stride;
  auto* g = reinterpret_cast<typename T::raw*>(a.grad) + (size_t)row * a.grad_stride;
  const int from = chunk * kDistillChunk;
  float v[kPer / 8][8];
#pragma unroll
  for (int i = 0; i < kPer / 8; ++i) {
    const int at = from + 8 * (i * kThreads + tid);
    load_part<T>(z + at, a.vocab - at, v[i]);
  }
  // p = 2^((z - m) c - less)
  float m, less;
  if constexpr (OWN_SUM) {
    m = a.row_sum[2 * row];
    less = a.row_sum[2 * row + 1];
  } else {
    const double sum = (double)a.lse[row] * (double)a.temperature;
    m = (float)sum;
    less = (float)((sum - (double)m) * (double)a.c);
  }
  if (tid < 64) {
    const Entries e = entries_of(a, row, tid);
#pragma unroll
    for (int i = 0; i < kMaxK / 64; ++i)
      entry[64 * i + tid] = {e.index[i] - from, e.index[i] >= 0 ? (float)(e.w[i] / e.total) : 0.f};
    if (tid == 0) some = e.any;
  }
#pragma unroll
  for (int i = 0; i < kPer / 4; ++i) *reinterpret_cast<float4*>(&share[4 * (i * kThreads + tid)]) = make_float4(0.f, 0.f, 0.f, 0.f);
  __syncthreads();
  for (int k = tid; k < a.k; k += kThreads) {
    const int at = entry[k].index;
    if ((uint32_t)at >= (uint32_t)kDistillChunk || entry[k].q == 0.f) continue;
    // the first entry of a place adds up all of them
    bool first = true;
    float q = 0.f;
    for (int o = 0; o < a.k; ++o) {
      if (entry[o].index != at) continue;
      first &= o >= k || entry[o].q == 0.f;
      q += entry[o].q;
    }
    if (first) share[at] = q;
  }
  __syncthreads();
  const float f = some ? a.temperature * (a.grad_loss ? a.grad_loss[row] : 1.f) : 0.f;
#pragma unroll
  for (int i = 0; i < kPer / 8; ++i) {
    const int at = 8 * (i * kThreads + tid), n = a.vocab - from - at;
    float o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float p = v[i][j] == -__builtin_inff() ? 0.f : power(v[i][j] - m, a, less);
      o[j] = f == 0.f ? 0.f : f * (p - share[at + j]);
    }
    store8<T>(g + from + at, n, o);
  }
}

template <class T>
int launch_type(const DistillArgs& a, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  const dim3 chunks(a.rows * a.nchunk), block(kThreads);
  if (a.loss) {
    hipLaunchKernelGGL(distill_sums_kernel<T>, chunks, block, 0, st, a);
    hipLaunchKernelGGL(distill_loss_kernel<T>, dim3((a.rows + kThreads / 64 - 1) / (kThreads / 64)), block, 0, st, a);
    if (a.grad) hipLaunchKernelGGL((distill_grad_kernel<T, true>), chunks, block, 0, st, a);
  } else {
    hipLaunchKernelGGL((distill_grad_kernel<T, false>), chunks, block, 0, st, a);
  }
  return (int)hipGetLastError();
}

}  // namespace

int launch_distill(const DistillArgs& a, int type, void* stream) {
  switch (type) {
    case 0: return launch_type<F32>(a, stream);
    case 1: return launch_type<F16>(a, stream);
    case 2: return launch_type<BF16>(a, stream);
    default: return (int)hipErrorInvalidValue;
  }
}

}  // namespace kvq
