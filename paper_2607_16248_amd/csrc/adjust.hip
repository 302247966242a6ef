// Penalties for repeated tokens, biases and masks on rows of logits (gfx950;
// include/dgap.h states them).
//
//   out_t = masked ? -inf : pen(z_t) - (f n_t + p [n_t > 0]) + bias_t,
//   pen(z) = seen_t ? (z > 0 ? z / r : z r) : z
//
// Bound by memory: every logit is read and written once.  A workgroup takes
// kAdjustChunk logits of a row.  It counts the row's history in a table of its
// own chunk in LDS (a word per logit: the number of times it was generated, and
// a bit for "seen"), so every workgroup of a row reads the whole history, which
// the caches hold; integer additions, so no order shows.  Its logits are asked
// for before that.  Biases name their tokens in a second table (the largest entry
// number wins), present where the call has any.
#include <hip/hip_runtime.h>

#include "decode_common.h"
#include "kvq_internal.h"
#include "logits_common.h"

namespace kvq {
namespace {

using namespace logits;

constexpr int kThreads = 256;
constexpr int kRuns = kAdjustChunk / (8 * kThreads);  // runs of 8 logits per thread
constexpr uint32_t kSeen = 0x80000000u;               // below it: generated, at most 2^24 times

template <class T, bool BIAS, bool RUNS>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs a) {
  using raw = typename T::raw;
  __shared__ __attribute__((aligned(16))) uint32_t count[kAdjustChunk];
  __shared__ __attribute__((aligned(16))) uint32_t slot[BIAS ? kAdjustChunk : 4];
  const int row = blockIdx.x / a.nchunk, chunk = blockIdx.x - row * a.nchunk, tid = threadIdx.x;
  const raw* in = reinterpret_cast<const raw*>(a.logits) + (int64_t)row * a.row_stride;
  raw* out = reinterpret_cast<raw*>(a.out) + (int64_t)row * a.out_stride;
  // RUNS: chunks begin where 16 bytes do, up to 7 logits before the row
  const int shift = RUNS ? (int)((reinterpret_cast<uintptr_t>(in) / sizeof(raw)) & 7) : 0;
  const int base = chunk * kAdjustChunk - shift;  // the chunk's first logit
  if (base >= a.vocab) return;

  // logit of place (i, j): run i of the thread, element j of the run
  auto place = [&](int i, int j) { return RUNS ? 8 * (i * kThreads + tid) + j : (8 * i + j) * kThreads + tid; };
  raw8_t<T> x[kRuns];
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int t0 = base + place(i, 0);
    if (RUNS && t0 >= 0 && t0 + 8 <= a.vocab) {
      x[i] = *reinterpret_cast<const raw8_t<T>*>(in + t0);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int t = base + place(i, j);
        x[i][j] = t >= 0 && t < a.vocab ? in[t] : T::make(0.f);
      }
    }
  }

  const float r = a.repetition ? a.repetition[row] : 1.f, p = a.presence ? a.presence[row] : 0.f,
              f = a.frequency ? a.frequency[row] : 0.f;
  const bool bad = !(r > 0.f) || !__builtin_isfinite(r) || !__builtin_isfinite(p) || !__builtin_isfinite(f);
  for (int k = tid * 4; k < kAdjustChunk; k += 4 * kThreads) {
    *reinterpret_cast<uint4*>(count + k) = make_uint4(0u, 0u, 0u, 0u);
    if constexpr (BIAS) *reinterpret_cast<uint4*>(slot + k) = make_uint4(0u, 0u, 0u, 0u);
  }
  __syncthreads();
  if (a.tokens) {
    const int n = a.length ? min(max(a.length[row], 0), a.history) : a.history;
    const int given = a.prompt ? a.prompt[row] : 0;
    const int32_t* h = a.tokens + (int64_t)row * a.history;
    const uint32_t end = (uint32_t)min(kAdjustChunk, a.vocab - base);
    constexpr int kAhead = 8;
    for (int k0 = tid; k0 < n; k0 += kAhead * kThreads) {
      int t[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) t[u] = k0 + u * kThreads < n ? h[k0 + u * kThreads] : -1;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const uint32_t at = (uint32_t)t[u] - (uint32_t)base;
        if (t[u] < 0 || at >= end) continue;
        if (k0 + u * kThreads < given) atomicOr(count + at, kSeen);
        else atomicAdd(count + at, 1u);
      }
    }
  }
  if constexpr (BIAS) {
    const uint32_t end = (uint32_t)min(kAdjustChunk, a.vocab - base);
    for (int k = tid; k < a.biases; k += kThreads) {
      const int t = a.bias_token[(int64_t)row * a.biases + k];
      const uint32_t at = (uint32_t)t - (uint32_t)base;
      if (t >= 0 && at < end) atomicMax(slot + at, (uint32_t)k + 1u);
    }
  }
  __syncthreads();

  const uint32_t* bits = nullptr;
  if (a.mask) {
    const int m = a.mask_row ? a.mask_row[row] : row;
    if (m >= 0 && m < a.mask_rows) bits = a.mask + (int64_t)m * a.mask_stride;
  }
  auto adjusted = [&](raw z0, int at, bool allowed) -> raw {
    const uint32_t c = count[at];
    uint32_t s = 0u;
    if constexpr (BIAS) s = slot[at];
    raw o = z0;
    if ((c | s) != 0u) {
      float z = T::value(z0);
      if (c != 0u && r != 1.f) z = z > 0.f ? z / r : z * r;
      const uint32_t n = c & ~kSeen;
      if (n != 0u) z -= fmaf(f, (float)n, p);
      if (BIAS && s != 0u) {
        const float b = a.bias[(int64_t)row * a.biases + (s - 1u)];
        z = b == -__builtin_inff() ? b : z + b;
      }
      o = T::make(z);
    }
    if (!allowed) o = T::make(-__builtin_inff());
    if (bad) o = T::make(__builtin_nanf(""));
    return o;
  };
  const int words = (a.vocab + 31) / 32;
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int t0 = base + place(i, 0);
    if (RUNS && t0 >= 0 && t0 + 8 <= a.vocab) {
      uint32_t allow = 0xFFu;
      if (bits) {
        const uint32_t w0 = bits[t0 >> 5], w1 = bits[min((t0 >> 5) + 1, words - 1)];
        allow = (uint32_t)((((uint64_t)w1 << 32) | w0) >> (t0 & 31));
      }
      raw8_t<T> o;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = adjusted(x[i][j], place(i, j), (allow >> j) & 1u);
      *reinterpret_cast<raw8_t<T>*>(out + t0) = o;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int t = base + place(i, j);
        if (t < 0 || t >= a.vocab) continue;
        out[t] = adjusted(x[i][j], place(i, j), !bits || ((bits[t >> 5] >> (t & 31)) & 1u));
      }
    }
  }
}

template <class T>
int launch_type(const AdjustArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.batch * a.nchunk)), block(kThreads);
  if (a.biases > 0) {
    if (a.runs) hipLaunchKernelGGL((adjust_kernel<T, true, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((adjust_kernel<T, true, false>), grid, block, 0, s, a);
  } else {
    if (a.runs) hipLaunchKernelGGL((adjust_kernel<T, false, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((adjust_kernel<T, false, false>), grid, block, 0, s, a);
  }
  return (int)hipGetLastError();
}

}  // namespace

int launch_adjust(const AdjustArgs& a, int type, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  switch (type) {
    case 0: return launch_type<F32>(a, s);
    case 1: return launch_type<F16>(a, s);
    case 2: return launch_type<BF16>(a, s);
    default: return (int)hipErrorInvalidValue;
  }
}

}  // namespace kvq
