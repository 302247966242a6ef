// Penalties for repeated tokens, biases and masks on rows of logits (gfx950;
// include/dgap.h states them).
//
//   out_t = masked ? -inf : pen(z_t) - (f n_t + p [n_t > 0]) + bias_t,
//   pen(z) = seen_t ? (z > 0 ? z / r : z r) : z
//
// Bound by memory: every logit is read and written once.  A workgroup takes a chunk of
// logits of a row and asks for them and their mask bits first.  It counts the row's
// history in a table of its own chunk in LDS (a word per logit), so every workgroup of a
// row reads the whole history, which the caches hold; integer additions, so no order
// shows.  Biases name their entries in the same word (the largest entry number wins); with
// a second table for them fewer workgroups fit (64 rows of 152064 bf16 under masks: 21 us
// to 15).  512 rows of 128256 fp16: 53 us without a history (4.9 TB/s), 62 with 1024
// tokens, 77 with 8192.  Listing the touched logits, so that a lane takes one each, and
// leaving the others alone was slower: 67 and 99.
#include <hip/hip_runtime.h>

#include "decode_common.h"
#include "kvq_internal.h"
#include "logits_common.h"

namespace kvq {
namespace {

using namespace logits;

// The table's word of a logit.  Packed: bits 0 to 14 count, bit 15 says "seen", the upper
// half is the bias entry; wide: bits 0 to 24 count, bit 31 "seen", the entry in a second
// table.
template <bool WIDE>
constexpr uint32_t kSeen = WIDE ? 0x80000000u : 0x8000u;

template <class T, int CHUNK, bool WIDE, bool RUNS>
__global__ __launch_bounds__(CHUNK / kAdjustPerThread) void adjust_kernel(AdjustArgs a) {
  constexpr int kThreads = CHUNK / kAdjustPerThread, kRuns = kAdjustPerThread / 8;  // runs of 8 logits per thread
  using raw = typename T::raw;
  __shared__ __attribute__((aligned(16))) uint32_t count[CHUNK];
  __shared__ __attribute__((aligned(16))) uint32_t slot[WIDE ? CHUNK : 4];
  const int row = blockIdx.x / a.nchunk, chunk = blockIdx.x - row * a.nchunk, tid = threadIdx.x;
  const raw* in = reinterpret_cast<const raw*>(a.logits) + (int64_t)row * a.row_stride;
  raw* out = reinterpret_cast<raw*>(a.out) + (int64_t)row * a.out_stride;
  // RUNS: chunks begin where 16 bytes do, up to 7 logits before the row
  const int shift = RUNS ? (int)((reinterpret_cast<uintptr_t>(in) / sizeof(raw)) & 7) : 0;
  const int base = chunk * CHUNK - shift;  // the chunk's first logit
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

  const uint32_t* bits = nullptr;
  if (a.mask) {
    const int m = a.mask_row ? a.mask_row[row] : row;
    if (m >= 0 && m < a.mask_rows) bits = a.mask + (int64_t)m * a.mask_stride;
  }
  const int words = (a.vocab + 31) / 32;
  uint2 allow[kRuns];  // the words that hold a run's bits
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int t0 = base + place(i, 0);
    allow[i] = make_uint2(~0u, ~0u);
    if (RUNS && bits && t0 >= 0 && t0 + 8 <= a.vocab)
      allow[i] = make_uint2(bits[t0 >> 5], bits[min((t0 >> 5) + 1, words - 1)]);
  }
  const float r = a.repetition ? a.repetition[row] : 1.f, p = a.presence ? a.presence[row] : 0.f,
              f = a.frequency ? a.frequency[row] : 0.f;
  const bool bad = !(r > 0.f) || !__builtin_isfinite(r) || !__builtin_isfinite(p) || !__builtin_isfinite(f);
  for (int k = tid * 4; k < CHUNK; k += 4 * kThreads) {
    *reinterpret_cast<uint4*>(count + k) = make_uint4(0u, 0u, 0u, 0u);
    if constexpr (WIDE) *reinterpret_cast<uint4*>(slot + k) = make_uint4(0u, 0u, 0u, 0u);
  }
  __syncthreads();
  if (a.tokens) {
    const int n = a.length ? min(max(a.length[row], 0), a.history) : a.history;
    const int given = a.prompt ? a.prompt[row] : 0;
    const int32_t* h = a.tokens + (int64_t)row * a.history;
    const uint32_t end = (uint32_t)min(CHUNK, a.vocab - base);
    constexpr int kAhead = 8;
    for (int k0 = tid; k0 < n; k0 += kAhead * kThreads) {
      int t[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) t[u] = k0 + u * kThreads < n ? h[k0 + u * kThreads] : -1;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const uint32_t at = (uint32_t)t[u] - (uint32_t)base;
        if (t[u] < 0 || at >= end) continue;
        if (k0 + u * kThreads < given) atomicOr(count + at, kSeen<WIDE>);
        else atomicAdd(count + at, 1u);
      }
    }
  }
  if (a.biases > 0) {
    const uint32_t end = (uint32_t)min(CHUNK, a.vocab - base);
    if constexpr (!WIDE) __syncthreads();  // (the lower halves stand from here on)
    for (int k = tid; k < a.biases; k += kThreads) {
      const int t = a.bias_token[(int64_t)row * a.biases + k];
      const uint32_t at = (uint32_t)t - (uint32_t)base;
      if (t < 0 || at >= end) continue;
      if constexpr (WIDE) atomicMax(slot + at, (uint32_t)k + 1u);
      else atomicMax(count + at, ((uint32_t)k + 1u) << 16 | (count[at] & 0xFFFFu));
    }
  }
  __syncthreads();

  auto adjusted = [&](raw z0, int at, bool allowed) -> raw {
    const uint32_t word = count[at];
    const uint32_t c = WIDE ? word : word & 0xFFFFu, s = WIDE ? slot[at] : word >> 16;
    raw o = z0;
    if ((c | s) != 0u) {
      float z = T::value(z0);
      if (c != 0u && r != 1.f) z = z > 0.f ? z / r : z * r;
      const uint32_t n = c & ~kSeen<WIDE>;
      if (n != 0u) z -= fmaf(f, (float)n, p);
      if (s != 0u) {
        const float b = a.bias[(int64_t)row * a.biases + (s - 1u)];
        z = b == -__builtin_inff() ? b : z + b;
      }
      o = T::make(z);
    }
    if (!allowed) o = T::make(-__builtin_inff());
    if (bad) o = T::make(__builtin_nanf(""));
    return o;
  };
#pragma unroll
  for (int i = 0; i < kRuns; ++i) {
    const int t0 = base + place(i, 0);
    if (RUNS && t0 >= 0 && t0 + 8 <= a.vocab) {
      const uint32_t eight = (uint32_t)((((uint64_t)allow[i].y << 32) | allow[i].x) >> (t0 & 31));
      raw8_t<T> o;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = adjusted(x[i][j], place(i, j), (eight >> j) & 1u);
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

template <class T, int CHUNK, bool WIDE>
int launch_chunks(const AdjustArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.batch * a.nchunk)), block(CHUNK / kAdjustPerThread);
  if (a.runs) hipLaunchKernelGGL((adjust_kernel<T, CHUNK, WIDE, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((adjust_kernel<T, CHUNK, WIDE, false>), grid, block, 0, s, a);
  return (int)hipGetLastError();
}

template <class T>
int launch_type(const AdjustArgs& a, hipStream_t s) {
  if (a.wide) return launch_chunks<T, kAdjustChunk, true>(a, s);
  return a.chunk == kAdjustLong ? launch_chunks<T, kAdjustLong, false>(a, s) : launch_chunks<T, kAdjustChunk, false>(a, s);
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
