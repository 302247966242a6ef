// The loss of a student's logits against a teacher's top logits, and its
// gradient (gfx950; include/dgap.h states both).
//
//   loss_r = T^2 sum_k q_k (log q_k - log p_{i_k}),  p = softmax(z / T) over the
//   vocabulary, q = softmax(t / T) over the row's entries;
//   d loss_r / d z_j = T (p_j - sum_k q_k [i_k = j]).
//
// Bound by memory: the loss reads every logit once, the gradient writes each once
// more (and reads it again where the row did not stay in registers).
// Exponentials in base 2, c = log2(e) / T, of differences to the row's largest logit.
//   row     workgroups of 1024 threads, each with a row in its registers (up to
//           163840 logits of 16 bits, 65536 of 32) and one row after the other: every
//           logit is read once
//   sums, loss, grad   for the loss alone, calls that the cache holds, and rows that
//           do not fit: one workgroup per (row, chunk) for sums and gradient, one
//           wave per row for the loss; the gradient reads the logits again
// Measured, 4096 rows of 128256 bf16, 64 entries: row 441 us, 4.8 TB/s of logits and
// gradient (a copy moves 4.9), three launches 600.  With one row per workgroup at a
// time, loads, sums and stores one after the other, the row kernel took 580; its
// arithmetic (two exponentials and a dozen instructions per logit, about 18 us per
// row and compute unit) shows wherever it does not run beside the loads.  The
// gradient alone of 4096 rows moves 5.4 TB/s (388 us), of 512, which the cache holds,
// 6.3 (41.5 us); with a table of fp32 shares per chunk, cleared
// and scattered to, it moved 3.
// The teacher's entries reach the gradient through a table of the runs of 8 logits
// that a thread handles: a run's first entry, from there the next one's number.
// Entries of one index are added in their order beforehand, so no sum depends on
// timing, every value is written once, and the gradient may take the logits' place.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "decode_common.h"
#include "kvq_internal.h"
#include "logits_common.h"

namespace kvq {
namespace {

using namespace logits;

constexpr int kThreads = 256;
constexpr int kPer = kDistillChunk / kThreads;  // logits per thread, in runs of 8
constexpr int kMaxK = kDistillMaxK;
constexpr int kRowThreads = 1024;
constexpr float kLowest = -3.402823466e38f;

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

// 2^(x c), x a difference to the row's largest logit: taken before c, so that
// neither the type's lowest value nor a whole row of it overflows; -inf gives 0.  c
// in fp32 moves an exponent by 2^-25 of itself, a weight by no more than 2^-25.
__device__ __forceinline__ float power(float x, const DistillArgs& a) { return __builtin_amdgcn_exp2f(x * a.c); }

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
  m = fmaxf(m, kLowest);  // (nothing but -inf: sums of 0)
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kPer / 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) s += power(v[i][j] - m, a);
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

// The row's entries, up to kMaxK / 64 per lane of a wave: places (-1: none),
// base-2 logits x = (t - max) c, shares q = 2^x / total, the student's logits z.
struct Entries {
  int index[kMaxK / 64];
  float x[kMaxK / 64], q[kMaxK / 64], z[kMaxK / 64];
  float total;
  bool any;
};
template <class T>
__device__ __forceinline__ Entries entries_of(const DistillArgs& a, int row, int lane) {
  const auto* z = reinterpret_cast<const typename T::raw*>(a.logits) + (size_t)row * a.row_stride;
  Entries e;
  float t[kMaxK / 64], top = -__builtin_inff();
  bool some = false;
#pragma unroll
  for (int i = 0; i < kMaxK / 64; ++i) {
    const int k = 64 * i + lane;
    e.index[i] = k < a.k ? a.index[(size_t)row * a.k + k] : -1;
    t[i] = k < a.k ? a.teacher[(size_t)row * a.k + k] : -__builtin_inff();
    if ((uint32_t)e.index[i] >= (uint32_t)a.vocab || t[i] == -__builtin_inff()) e.index[i] = -1;
    e.z[i] = a.loss && e.index[i] >= 0 ? T::value(z[e.index[i]]) : 0.f;
    if (e.index[i] >= 0) {
      top = fmaxf(top, t[i]);
      some = true;
    }
  }
  top = dec::wave_max(top);
  e.any = __builtin_amdgcn_ballot_w64(some) != 0;  // (a NaN is an entry, which no maximum shows)
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < kMaxK / 64; ++i) {
    e.x[i] = (t[i] - top) * a.c;
    e.q[i] = e.index[i] >= 0 ? power(t[i] - top, a) : 0.f;
    sum += e.q[i];
  }
  e.total = dec::wave_sum(sum);
#pragma unroll
  for (int i = 0; i < kMaxK / 64; ++i) e.q[i] = e.any ? e.q[i] / e.total : 0.f;
  return e;
}

// One wave: the row's loss, with its largest logit m and log_sum = log2 of the
// sum of 2^((z - m) c).  The logarithms and their sum are in 64 bits.
__device__ __forceinline__ float loss_of(const DistillArgs& a, const Entries& e, float m, double log_sum) {
  const double c = (double)a.c, log_total = e.any ? log2((double)e.total) : 0.0;
  double loss = 0.0;
#pragma unroll
  for (int i = 0; i < kMaxK / 64; ++i)
    if (e.index[i] >= 0 && !(e.q[i] == 0.f))  // (NaN: a teacher logit of NaN or +inf)
      loss += (double)e.q[i] * ((double)e.x[i] - log_total - ((double)e.z[i] - (double)m) * c + log_sum);
  return (float)(wave_sum_d(loss) * 0.6931471805599453 * (double)a.temperature * (double)a.temperature);
}

// The entries of the runs of 8 logits of a chunk (or a row), in LDS: head[run / 2]
// is 0 or 1 + an entry of the two runs, next that entry's next one of them.
template <int RUNS>
struct Shares {
  uint32_t head[RUNS / 2];
  int index[kMaxK];
  float q[kMaxK], sum[kMaxK];  // an entry's share; that of all of its index
  uint32_t next[kMaxK];
  int some;
};
template <int NT, int RUNS>
__device__ __forceinline__ void clear_shares(Shares<RUNS>& s) {
  for (int i = threadIdx.x; i < RUNS / 2; i += NT) s.head[i] = 0;
}
// wave 0 puts the row's entries, as places from `from` on
template <int RUNS>
__device__ __forceinline__ void put_entries(Shares<RUNS>& s, const Entries& e, int from, int lane) {
#pragma unroll
  for (int i = 0; i < kMaxK / 64; ++i) {
    s.index[64 * i + lane] = e.index[i] >= 0 && e.q[i] != 0.f ? e.index[i] - from : -1;
    s.q[64 * i + lane] = e.q[i];
  }
  if (lane == 0) s.some = e.any;
}
// After a barrier every entry's thread links it to its run (the order within a
// run is any), and after another one finds what its index adds up to: the first
// entry of an index the sum of all of them in their order, the others 0.
template <int NT, int RUNS>
__device__ __forceinline__ void link_shares(Shares<RUNS>& s, int count) {
  for (int k = threadIdx.x; k < count; k += NT) {
    const int at = s.index[k];
    if ((uint32_t)at < 8u * RUNS) s.next[k] = atomicExch(&s.head[at >> 4], 1u + k);
  }
}
template <int NT, int RUNS>
__device__ __forceinline__ void sum_shares(Shares<RUNS>& s, int count) {
  for (int k = threadIdx.x; k < count; k += NT) {
    const int at = s.index[k];
    if ((uint32_t)at >= 8u * RUNS) continue;
    bool first = true, more = false;
    for (uint32_t e = s.head[at >> 4]; e != 0; e = s.next[e - 1]) {
      const bool same = s.index[e - 1] == at && (int)e - 1 != k;
      more |= same;
      first &= !same || (int)e - 1 > k;
    }
    float q = s.q[k];
    if (more && first)
      for (int o = k + 1; o < count; ++o) q += s.index[o] == at ? s.q[o] : 0.f;
    s.sum[k] = first ? q : 0.f;
  }
}
// The gradient f (p - share) of a run of 8 logits x, p = 2^((x - m) c) r.
struct Softmax {
  float m, r;
};
template <class T, int RUNS>
__device__ __forceinline__ raw8_t<T> grad_of(const DistillArgs& a, const Shares<RUNS>& s, const raw8_t<T>& x, int run,
                                             const Softmax& p, float f) {
  float g[8];
  const float fr = f * p.r;
#pragma unroll
  for (int j = 0; j < 8; ++j) g[j] = fr * power(T::value(x[j]) - p.m, a);
  for (uint32_t e = s.head[run >> 1]; e != 0; e = s.next[e - 1]) {
    const int at = s.index[e - 1] - 8 * run;
    const float q = s.sum[e - 1];
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = j == at ? fmaf(-f, q, g[j]) : g[j];
  }
  raw8_t<T> o;
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = T::make(g[j]);
  return o;
}
// of the last few logits, one a thread
template <class T, int RUNS>
__device__ __forceinline__ typename T::raw grad_one(const DistillArgs& a, const Shares<RUNS>& s, float v, int at, const Softmax& p, float f) {
  raw8_t<T> x = all8<T>(-__builtin_inff());
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = j == (at & 7) ? T::make(v) : x[j];
  const raw8_t<T> o = grad_of<T>(a, s, x, at >> 3, p, f);
  typename T::raw r = o[0];
#pragma unroll
  for (int j = 1; j < 8; ++j) r = j == (at & 7) ? o[j] : r;
  return r;
}
// That of a row without entries, whose gradient is 0 also where nothing in it is
// finite: every logit, -inf too, gives 0 times a power of at most 1.
constexpr Softmax kNoEntries = {3.402823466e38f, 0.f};
// From the caller's log-sum-exp: m its place among the logits, as near as fp32
// has it, and r what that leaves.
__device__ __forceinline__ Softmax from_lse(const DistillArgs& a, int row) {
  const double sum = (double)a.lse[row] * (double)a.temperature;
  const float m = (float)sum;
  return {m, __builtin_amdgcn_exp2f((float)(((double)m - sum) * (double)a.c))};
}
template <class T>
__device__ __forceinline__ void store8(typename T::raw* p, const raw8_t<T>& x) {
  typedef raw8_t<T> any __attribute__((aligned(sizeof(typename T::raw))));
  *reinterpret_cast<any*>(p) = x;
}

template <class T>
__global__ __launch_bounds__(kThreads) void distill_loss_kernel(DistillArgs a) {
  const int row = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= a.rows) return;
  const float* part = a.ws + (size_t)row * a.nchunk * 2;
  const double c = (double)a.c;
  float m = -__builtin_inff();
  for (int i = lane; i < a.nchunk; i += 64) m = fmaxf(m, part[2 * i]);
  m = dec::wave_max(m);
  double s = 0.0;
  for (int i = lane; i < a.nchunk; i += 64)
    if (part[2 * i + 1] != 0.f) s += (double)part[2 * i + 1] * exp2(((double)part[2 * i] - (double)m) * c);
  const double sum = wave_sum_d(s), log_sum = log2(sum);  // of 2^((z - m) c)
  const float loss = loss_of(a, entries_of<T>(a, row, lane), m, log_sum);
  if (lane == 0) {
    a.loss[row] = loss;
    if (a.lse) a.lse[row] = (float)((log_sum + (double)m * c) * 0.6931471805599453);
    if (a.grad) {  // for the gradient's launch
      a.row_sum[2 * row] = m;
      a.row_sum[2 * row + 1] = (float)(1.0 / sum);
    }
  }
}

// OWN_SUM: with what distill_loss_kernel left, else from the caller's lse
template <class T, bool OWN_SUM>
__global__ __launch_bounds__(kThreads) void distill_grad_kernel(DistillArgs a) {
  __shared__ Shares<kDistillChunk / 8> s;
  const int row = blockIdx.x / a.nchunk, chunk = blockIdx.x % a.nchunk, tid = threadIdx.x;
  const auto* z = reinterpret_cast<const typename T::raw*>(a.logits) + (size_t)row * a.row_stride;
  auto* g = reinterpret_cast<typename T::raw*>(a.grad) + (size_t)row * a.grad_stride;
  const int from = chunk * kDistillChunk, count = min(kDistillChunk, a.vocab - from), bulk = count & ~7;
  raw8_t<T> v[kPer / 8];
  if (bulk > 0) {
#pragma unroll
    for (int i = 0; i < kPer / 8; ++i) v[i] = load8<T>(z + from + min(8 * (i * kThreads + tid), bulk - 8));
  }
  Softmax p = OWN_SUM ? Softmax{a.row_sum[2 * row], a.row_sum[2 * row + 1]} : from_lse(a, row);
  if (tid < 64) put_entries(s, entries_of<T>(a, row, tid), from, tid);
  clear_shares<kThreads>(s);
  __syncthreads();
  link_shares<kThreads>(s, a.k);
  __syncthreads();
  sum_shares<kThreads>(s, a.k);
  __syncthreads();
  if (!s.some) p = kNoEntries;
  const float f = s.some ? a.temperature * (a.grad_loss ? a.grad_loss[row] : 1.f) : 0.f;
  // (a run past the end was loaded as the last one, which its own thread may
  // have written by now: it is not used)
#pragma unroll
  for (int i = 0; i < kPer / 8; ++i) {
    const int run = i * kThreads + tid;
    if (8 * run < bulk) store8<T>(g + from + 8 * run, grad_of<T>(a, s, v[i], run, p, f));
  }
  if (bulk + tid < count) g[from + bulk + tid] = grad_one<T>(a, s, T::value(z[from + bulk + tid]), bulk + tid, p, f);
}

// The run as it is, with no memory of what was made of it: its fp32 values would
// else be kept from one pass over the row to the next (88 to 170 registers spilled).
template <class T>
__device__ __forceinline__ void forget(raw8_t<T>& v) {
  typedef uint32_t words __attribute__((ext_vector_type(sizeof(raw8_t<T>) / 4)));
  words w = __builtin_bit_cast(words, v);
#pragma unroll
  for (int i = 0; i < (int)(sizeof(raw8_t<T>) / 4); ++i) {
    uint32_t x = w[i];
    asm volatile("" : "+v"(x));
    w[i] = x;
  }
  v = __builtin_bit_cast(raw8_t<T>, w);
}

// Rows in the registers of one workgroup, one after the other, RUNS runs of 8
// logits per thread.  As soon as a run's gradient is stored its registers take the
// next row's, which joins the thread's running maximum and sum some runs later:
// loads, stores and arithmetic go on together, and a row ends in one reduction of
// the threads' sums.  The next row's entries are linked meanwhile.
template <class T, int RUNS>
__global__ __launch_bounds__(kRowThreads) void distill_row_kernel(DistillArgs a) {
  constexpr int kWaves = kRowThreads / 64, kBehind = RUNS / 4;
  __shared__ Shares<RUNS * kRowThreads> shares[2];
  __shared__ Entries held[2][64];  // wave 0's, until the loss
  __shared__ float part[2][kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, bulk = a.vocab & ~7;
  const bool has_last = bulk + tid < a.vocab;
  raw8_t<T> v[RUNS];
  float last, m = kLowest, sum = 0.f;  // the last few logits, one a thread; the incoming row's maximum and sum
  auto own_run = [&](int i) {
    uint32_t run = i * kRowThreads + tid;
    asm volatile("" : "+v"(run));  // (or every run keeps its places in registers)
    return (int)run;
  };
  auto load = [&](int row, int i) {
    const auto* z = reinterpret_cast<const typename T::raw*>(a.logits) + (size_t)row * a.row_stride;
    v[i] = load8<T>(z + min(8 * own_run(i), bulk - 8));
  };
  auto load_last = [&](int row) {
    const auto* z = reinterpret_cast<const typename T::raw*>(a.logits) + (size_t)row * a.row_stride;
    last = has_last ? T::value(z[bulk + tid]) : -__builtin_inff();
  };
  auto join = [&](float top, float other) {  // another part's maximum and sum
    const float n = fmaxf(m, top);
    sum = sum * power(m - n, a) + other * power(top - n, a);
    m = n;
  };
  auto take = [&](int i) {  // run i of the incoming row
    forget<T>(v[i]);
    float x[8], top = kLowest, s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = T::value(v[i][j]);
      top = fmaxf(top, x[j]);
    }
    const float n = fmaxf(m, top);
#pragma unroll
    for (int j = 0; j < 8; ++j) s += power(x[j] - n, a);
    // (a run past the end repeats the last one: no matter to the maximum)
    sum = fmaf(sum, power(m - n, a), 8 * own_run(i) < bulk ? s : 0.f);
    m = n;
  };
  auto list = [&](int row, int buf) {
    clear_shares<kRowThreads>(shares[buf]);
    if (wv == 0) {
      const Entries e = entries_of<T>(a, row, lane);
      put_entries(shares[buf], e, 0, lane);
      held[buf][lane] = e;
    }
  };
#pragma unroll
  for (int i = 0; i < RUNS; ++i) load(blockIdx.x, i);
  load_last(blockIdx.x);
  list(blockIdx.x, 0);
  __syncthreads();
  link_shares<kRowThreads>(shares[0], a.k);
  __syncthreads();
  sum_shares<kRowThreads>(shares[0], a.k);
#pragma unroll
  for (int i = 0; i < RUNS; ++i) take(i);
  int buf = 0;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x, buf ^= 1) {
    if (has_last) join(fmaxf(last, kLowest), last == -__builtin_inff() ? 0.f : 1.f);
    const float top = dec::wave_max(m), all = dec::wave_sum(sum * power(m - top, a));
    if (lane == 0) {
      part[0][wv] = top;
      part[1][wv] = all;
    }
    __syncthreads();  // (and the row's shares are whole, the other ones free)
    Softmax p = {kLowest, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) p.m = fmaxf(p.m, part[0][w]);
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += part[1][w] * power(part[0][w] - p.m, a);
    p.r = 1.f / total;
    const auto& s = shares[buf];
    if (wv == 0) {
      const double log_sum = log2((double)total);
      const float loss = loss_of(a, held[buf][lane], p.m, log_sum);
      if (lane == 0) {
        a.loss[row] = loss;
        if (a.lse) a.lse[row] = (float)((log_sum + (double)p.m * (double)a.c) * 0.6931471805599453);
      }
    }
    if (!s.some) p = kNoEntries;
    const float f = s.some ? a.temperature * (a.grad_loss ? a.grad_loss[row] : 1.f) : 0.f;
    auto* g = reinterpret_cast<typename T::raw*>(a.grad) + (size_t)row * a.grad_stride;
    const int next = min(row + (int)gridDim.x, a.rows - 1);  // (after the last row: that one again, unused)
    if (has_last) g[bulk + tid] = grad_one<T>(a, s, last, bulk + tid, p, f);
    load_last(next);
    m = kLowest;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      const int run = own_run(i);
      forget<T>(v[i]);
      if (8 * run < bulk) store8<T>(g + 8 * run, grad_of<T>(a, s, v[i], run, p, f));
      load(next, i);
      if (i >= kBehind) take(i - kBehind);
      __builtin_amdgcn_sched_barrier(0);
      if (i == 0) list(next, buf ^ 1);
      if (i == RUNS / 4) {
        __syncthreads();
        link_shares<kRowThreads>(shares[buf ^ 1], a.k);
      }
      if (i == RUNS / 2) {
        __syncthreads();
        sum_shares<kRowThreads>(shares[buf ^ 1], a.k);
      }
    }
#pragma unroll
    for (int i = RUNS - kBehind; i < RUNS; ++i) take(i);
  }
}

template <class T, int RUNS>
int launch_row(const DistillArgs& a, hipStream_t st) {
  // (two workgroups of the smallest rows fit a compute unit)
  const dim3 grid(std::min(a.rows, a.compute_units * (RUNS * (int)sizeof(typename T::raw) <= 8 ? 2 : 1)));
  hipLaunchKernelGGL((distill_row_kernel<T, RUNS>), grid, dim3(kRowThreads), 0, st, a);
  return (int)hipGetLastError();
}

template <class T>
int launch_type(const DistillArgs& a, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  if (a.whole_rows) {
    // the fewest registers that hold the row
    const int runs = (a.vocab + 8 * kRowThreads - 1) / (8 * kRowThreads);
    if (runs <= 4) return launch_row<T, 4>(a, st);
    if (runs <= 8) return launch_row<T, 8>(a, st);
    if constexpr (sizeof(typename T::raw) == 2) {
      if (runs <= 16) return launch_row<T, 16>(a, st);
      if (runs <= 20) return launch_row<T, 20>(a, st);
    }
    return (int)hipErrorInvalidValue;
  }
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
