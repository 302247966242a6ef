// The next token of every row of logits (gfx950): temperature, top-k, top-p and
// min-p, one given uniform number per row (include/dgap.h states the rule).
//
// All filters keep a prefix of the row's descending order (equal logits by
// lower index), and the token is the element at which the kept mass, summed in
// that order, passes u times the kept total: every step is a search for the
// element where a count or a mass reaches a target.  With d = log2(e) / T
// (z_max - z) an element weighs 2^-d.
//   max     one workgroup per (row, chunk): the chunk's largest key
//   bins    one per (row, chunk): counts and masses of 2048 bins of d, 1/40 of an
//           octave each, added up per row with integer atomics
//   gather  one per (row, chunk): from the bins' prefix sums the bins where the
//           searches end (a bracket of bins, where a target depends on an
//           earlier search); their elements, a few hundred, go to the row's list
//   finish  one per row: the list sorted, the searches ended
// Masses are whole numbers of 2^-kUnit of the largest weight (64 bits): sums are
// exact, so they depend neither on the order of the atomics nor on which
// elements a bin or the list summed.  A weight is a 24-bit number (one hardware
// exponential of the fraction of d, taken in 64 bits); those below
// 2^-(kUnit + 1) count as 0, at most V 2^-(kUnit + 1) of the largest weight
// together.  They, and all of the last bin, are never chosen.
// A row whose bins hold more elements than a list (thousands of equal logits)
// is searched by the finish over all its logits, a digit of the keys at a time.
#include <hip/hip_runtime.h>

#include "kvq_internal.h"
#include "logits_common.h"

namespace kvq {
namespace {

using namespace logits;

constexpr int kThreads = 256;
constexpr int kBins = kSampleBins;
constexpr double kPerOctave = 40.0;  // 51 octaves: past them no weight is left (kUnit <= 45)
constexpr int kFinishThreads = 1024;
constexpr uint64_t kBadRow = ~0ull;  // key of a chunk that holds a NaN or +inf

struct Row {
  double inv;      // log2(e) / T
  float temperature, top_p, min_p, u;
  uint32_t k;      // elements that top-k keeps
  bool bad, greedy;
};
__device__ __forceinline__ bool not_finite(float x) { return !(__builtin_fabsf(x) < __builtin_inff()); }

__device__ __forceinline__ Row row_of(const SampleArgs& a, int row) {
  Row r;
  r.temperature = a.temperature ? a.temperature[row] : 1.f;
  const int k = a.top_k ? a.top_k[row] : 0;
  r.top_p = a.top_p ? a.top_p[row] : 1.f;
  r.min_p = a.min_p ? a.min_p[row] : 0.f;
  r.u = a.uniform[row];
  r.bad = not_finite(r.temperature) || r.temperature < 0.f || r.top_p != r.top_p || r.min_p != r.min_p || r.u != r.u;
  r.greedy = r.temperature == 0.f;
  r.inv = r.greedy ? 0.0 : 1.4426950408889634 / (double)r.temperature;
  r.k = k <= 0 || k > a.vocab ? (uint32_t)a.vocab : (uint32_t)k;
  if (r.min_p > 1.f) r.k = 1;  // only the largest logit
  r.u = fminf(fmaxf(r.u, 0.f), 0x1.fffffep-1f);
  return r;
}

__device__ __forceinline__ double depth(double zmax, float z, double inv) { return (zmax - (double)z) * inv; }
__device__ __forceinline__ int bin_of(double d) { return (int)fmin(d * kPerOctave, (double)(kBins - 1)); }
// 2^-d in units of 2^-unit
__device__ __forceinline__ uint64_t weight_of(double d, int unit) {
  if (!(d < (double)(unit + 1))) return 0;
  const int n = (int)d;
  const uint32_t m = (uint32_t)(__builtin_amdgcn_exp2f(-(float)(d - (double)n)) * 16777216.f);
  const int sh = unit - 24 - n;
  return sh >= 0 ? (uint64_t)m << sh : (uint64_t)((m + (1u << (-sh - 1))) >> -sh);
}

__device__ __forceinline__ uint64_t* row_mass(const SampleArgs& a, int row) {
  return reinterpret_cast<uint64_t*>(a.ws + (size_t)row * a.row_bytes);
}
__device__ __forceinline__ uint64_t* row_list(const SampleArgs& a, int row) { return row_mass(a, row) + kBins; }
__device__ __forceinline__ uint64_t* row_keys(const SampleArgs& a, int row) { return row_list(a, row) + kSampleList; }
__device__ __forceinline__ uint32_t* row_count(const SampleArgs& a, int row) {
  return reinterpret_cast<uint32_t*>(row_keys(a, row) + a.nchunk);  // [kBins], then the list's length
}

// f(logits, first index, valid) for the chunk's logits, 8 a thread at a time
template <class T, int NT, class F>
__device__ __forceinline__ void each8(const typename T::raw* z, int from, int to, F f) {
  for (int i = from + 8 * (int)threadIdx.x; i < to; i += 8 * NT) {
    float v[8];
    load8<T>(z + i, to - i, v);
    f(v, i, min(8, to - i));
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void sample_max_kernel(SampleArgs a) {
  __shared__ uint64_t part[kThreads / 64];
  const int row = blockIdx.x / a.nchunk, chunk = blockIdx.x % a.nchunk, tid = threadIdx.x;
  const auto* z = reinterpret_cast<const typename T::raw*>(a.logits) + (size_t)row * a.row_stride;
  // this workgroup's share of the row's bins and the list's length start at 0
  const int share = (kBins + a.nchunk - 1) / a.nchunk;
  for (int b = chunk * share + tid; b < min(kBins, (chunk + 1) * share); b += kThreads) {
    row_mass(a, row)[b] = 0;
    row_count(a, row)[b] = 0;
  }
  if (chunk == 0 && tid == 0) row_count(a, row)[kBins] = 0;
  uint64_t key = 0;
  const int from = chunk * kSampleChunk, to = min(a.vocab, from + kSampleChunk);
  each8<T, kThreads>(z, from, to, [&](const float(&v)[8], int i, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint64_t k = j < n ? make_key(v[j], i + j) : 0;
      if (!(v[j] < __builtin_inff())) k = kBadRow;
      key = k > key ? k : key;
    }
  });
  key = wave_max64(key);
  if ((tid & 63) == 0) part[tid >> 6] = key;
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) key = part[w] > key ? part[w] : key;
    row_keys(a, row)[chunk] = key;
  }
}

// The row's largest key, in every thread.
template <int NT>
__device__ __forceinline__ uint64_t row_top(const SampleArgs& a, int row, uint64_t* part) {
  uint64_t key = 0;
  for (int c = threadIdx.x; c < a.nchunk; c += NT) {
    const uint64_t k = row_keys(a, row)[c];
    key = k > key ? k : key;
  }
  key = wave_max64(key);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = key;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) key = part[w] > key ? part[w] : key;
  __syncthreads();
  return key;
}
// A row without a token to sample: settings out of range, NaN or +inf, nothing finite.
__device__ __forceinline__ bool no_token(const Row& r, uint64_t top) {
  return r.bad || top == kBadRow || !(key_value(top) > -__builtin_inff());
}

template <class T>
__global__ __launch_bounds__(kThreads) void sample_bins_kernel(SampleArgs a) {
  __shared__ uint64_t mass[kBins], part[kThreads / 64];
  __shared__ uint32_t count[kBins];
  const int row = blockIdx.x / a.nchunk, chunk = blockIdx.x % a.nchunk, tid = threadIdx.x;
  const Row r = row_of(a, row);
  if (r.bad || r.greedy) return;
  for (int b = tid; b < kBins; b += kThreads) {
    mass[b] = 0;
    count[b] = 0;
  }
  const uint64_t top = row_top<kThreads>(a, row, part);
  if (no_token(r, top)) return;
  const double zmax = (double)key_value(top);
  const auto* z = reinterpret_cast<const typename T::raw*>(a.logits) + (size_t)row * a.row_stride;
  const int from = chunk * kSampleChunk, to = min(a.vocab, from + kSampleChunk);
  uint32_t rest = 0;  // elements of the last bin
  each8<T, kThreads>(z, from, to, [&](const float(&v)[8], int, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= n) continue;
      const double d = depth(zmax, v[j], r.inv);
      const int b = bin_of(d);
      if (b == kBins - 1) {
        ++rest;
        continue;
      }
      atomicAdd(&count[b], 1u);
      atomicAdd(reinterpret_cast<unsigned long long*>(&mass[b]), (unsigned long long)weight_of(d, a.unit));
    }
  });
  if (rest) atomicAdd(&count[kBins - 1], rest);
  __syncthreads();
  for (int b = tid; b < kBins; b += kThreads) {
    if (count[b] == 0) continue;
    atomicAdd(&row_count(a, row)[b], count[b]);
    if (mass[b]) atomicAdd(reinterpret_cast<unsigned long long*>(&row_mass(a, row)[b]), (unsigned long long)mass[b]);
  }
}

// Where the searches of a row end, from its bins' prefix sums: top-k in bin kb
// (cut: inside it), top-p in one of the bins p0 .. p1, min-p in bin mb, the
// token in one of u0 .. u1.  A bin of -1 stands for no such search.
struct Ends {
  int kb, p0, p1, mb, u0, u1;
  bool cut;
  __device__ __forceinline__ bool wanted(int b) const {
    return (cut && b == kb) || (b >= p0 && b <= p1) || b == mb || (b >= u0 && b <= u1);
  }
};

// count[b], mass[b]: exclusive prefix sums over the bins (kBins + 1 of each).
struct Prefix {
  uint64_t mass[kBins + 1];
  uint32_t count[kBins + 1];
  uint64_t part[kFinishThreads / 64][2];
  int found[6];
};

template <int NT>
__device__ __forceinline__ Ends find_ends(const SampleArgs& a, int row, const Row& r, Prefix& s, uint32_t& wanted) {
  constexpr int kPer = kBins / NT;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  uint64_t m[kPer], msum = 0;
  uint32_t c[kPer], csum = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    m[j] = row_mass(a, row)[tid * kPer + j];
    c[j] = row_count(a, row)[tid * kPer + j];
    msum += m[j];
    csum += c[j];
  }
  const uint64_t mi = wave_scan64(msum), ci = wave_scan64(csum);
  if (lane == 63) {
    s.part[wv][0] = mi;
    s.part[wv][1] = ci;
  }
  if (tid < 6) s.found[tid] = -1;
  __syncthreads();
  uint64_t mb = mi - msum, cb = ci - csum;
  for (int w = 0; w < wv; ++w) {
    mb += s.part[w][0];
    cb += s.part[w][1];
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    s.mass[tid * kPer + j] = mb;
    s.count[tid * kPer + j] = (uint32_t)cb;
    mb += m[j];
    cb += c[j];
  }
  if (tid == NT - 1) {
    s.mass[kBins] = mb;
    s.count[kBins] = (uint32_t)cb;
  }
  __syncthreads();
  // the bin in which a test becomes true (test(b): it holds once bins 0 .. b - 1 are in)
  auto search = [&](int slot, auto test) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int b = tid * kPer + j;
      if (!test(b) && test(b + 1)) s.found[slot] = b;
    }
  };
  Ends e;
  search(0, [&](int b) { return s.count[b] >= r.k; });
  __syncthreads();
  e.kb = s.found[0];
  // (the last bin has no mass: it is never cut)
  e.cut = e.kb < kBins - 1 && s.count[e.kb + 1] != r.k;
  const double lo = (double)(e.cut ? s.mass[e.kb] : s.mass[e.kb + 1]), hi = (double)s.mass[e.kb + 1];
  e.p0 = e.p1 = -1;
  if (r.top_p < 1.f) {
    const double t0 = fmax((double)r.top_p * lo, 1.0), t1 = fmax((double)r.top_p * hi, 1.0);
    search(1, [&](int b) { return (double)s.mass[b] >= t0; });
    search(2, [&](int b) { return (double)s.mass[b] >= t1; });
    __syncthreads();
    e.p0 = s.found[1];
    e.p1 = s.found[2];
  }
  e.mb = -1;
  if (r.min_p > 0.f && r.min_p <= 1.f) {
    e.mb = bin_of(-log2((double)r.min_p));
    if (e.mb == kBins - 1) e.mb = -1;
  }
  int end0 = e.kb, end1 = e.kb;
  if (e.p0 >= 0) {
    end0 = min(end0, e.p0);
    end1 = min(end1, e.p1);
  }
  if (e.mb >= 0) {
    end0 = min(end0, e.mb);
    end1 = min(end1, e.mb);
  }
  const double t0 = (double)r.u * (double)s.mass[end0], t1 = (double)r.u * (double)s.mass[end1 + 1];
  search(3, [&](int b) { return (double)s.mass[b] > t0; });
  search(4, [&](int b) { return (double)s.mass[b] > t1; });
  __syncthreads();
  e.u0 = s.found[3];
  e.u1 = s.found[4];
  uint32_t own = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (e.wanted(tid * kPer + j)) own += c[j];
  const uint64_t all = wave_sum64(own);
  if (lane == 0) s.part[wv][0] = all;
  __syncthreads();
  wanted = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) wanted += (uint32_t)s.part[w][0];
  __syncthreads();
  return e;
}

template <class T>
__global__ __launch_bounds__(kThreads) void sample_gather_kernel(SampleArgs a) {
  __shared__ Prefix s;
  __shared__ uint64_t part[kThreads / 64];
  const int row = blockIdx.x / a.nchunk, chunk = blockIdx.x % a.nchunk;
  const Row r = row_of(a, row);
  if (r.bad || r.greedy) return;
  const uint64_t top = row_top<kThreads>(a, row, part);
  if (no_token(r, top)) return;
  uint32_t wanted;
  const Ends e = find_ends<kThreads>(a, row, r, s, wanted);
  if (wanted > (uint32_t)kSampleList) return;
  const double zmax = (double)key_value(top);
  const auto* z = reinterpret_cast<const typename T::raw*>(a.logits) + (size_t)row * a.row_stride;
  const int from = chunk * kSampleChunk, to = min(a.vocab, from + kSampleChunk);
  each8<T, kThreads>(z, from, to, [&](const float(&v)[8], int i, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= n || !e.wanted(bin_of(depth(zmax, v[j], r.inv)))) continue;
      const uint32_t at = atomicAdd(&row_count(a, row)[kBins], 1u);
      if (at < (uint32_t)kSampleList) row_list(a, row)[at] = make_key(v[j], i + j);
    }
  });
}

// A search over all of a row's logits, a digit of the keys at a time: the first
// element, in descending order, with which the count or the mass of the elements
// so far is past a target.
struct Found {
  uint64_t key, mass;  // the element; the mass up to and with it
};
struct Digits {
  uint64_t mass[256];
  uint32_t count[256];
  uint64_t before[2];
  uint32_t digit;
};
template <class T, class F>
__device__ Found search_row(const SampleArgs& a, const typename T::raw* z, double zmax, const Row& r, Digits& s, F past) {
  uint64_t prefix = 0, mass = 0, count = 0;
  // (bits 24-31, of the index's complement, are ones: V <= 2^24)
  for (int shift = 56; shift >= 0; shift -= 8) {
    if (shift == 24) {
      prefix = (prefix << 8) | 0xFFu;
      continue;
    }
    if (threadIdx.x < 256) {
      s.mass[threadIdx.x] = 0;
      s.count[threadIdx.x] = 0;
    }
    __syncthreads();
    for (int base = 0; base < a.vocab; base += 8 * kFinishThreads) {  // (every lane stays: waves add up together)
      const int i = base + 8 * (int)threadIdx.x, n = min(8, a.vocab - i);
      float v[8];
      load8<T>(z + i, n, v);
      uint32_t digit[8], first = 256, own = 0;
      uint64_t w[8], sum = 0;
      bool same = true;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint64_t key = make_key(v[j], i + j);
        const bool in = j < n && (shift == 56 || (key >> (shift + 8)) == prefix);
        digit[j] = in ? (uint32_t)(key >> shift) & 255u : 256u;
        w[j] = in ? weight_of(depth(zmax, v[j], r.inv), a.unit) : 0;
        if (!in) continue;
        first = first == 256 ? digit[j] : first;
        same &= digit[j] == first;
        ++own;
        sum += w[j];
      }
      const uint64_t some = __builtin_amdgcn_ballot_w64(own != 0);
      if (!some) continue;
      const uint32_t common = (uint32_t)__builtin_amdgcn_readlane((int)first, __builtin_ctzll(some));
      if (__builtin_amdgcn_ballot_w64(own != 0 && !(same && first == common)) == 0) {
        const uint64_t all = wave_sum64(sum), count_all = wave_sum64(own);
        if ((threadIdx.x & 63) == 0) {
          atomicAdd(&s.count[common], (uint32_t)count_all);
          atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[common]), (unsigned long long)all);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (digit[j] == 256) continue;
          atomicAdd(&s.count[digit[j]], 1u);
          atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[digit[j]]), (unsigned long long)w[j]);
        }
      }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      int d = 255;
      for (; d > 0; --d) {
        if (past(count + s.count[d], mass + s.mass[d])) break;
        count += s.count[d];
        mass += s.mass[d];
      }
      s.digit = (uint32_t)d;
      s.before[0] = count;
      s.before[1] = mass;
    }
    __syncthreads();
    count = s.before[0];
    mass = s.before[1];
    prefix = (prefix << 8) | s.digit;
    if (shift == 0) mass += s.mass[s.digit];
    __syncthreads();
  }
  return {prefix, mass};
}

template <class T>
__global__ __launch_bounds__(kFinishThreads) void sample_finish_kernel(SampleArgs a) {
  constexpr int kPer = kSampleList / kFinishThreads;
  __shared__ Prefix s;
  __shared__ uint64_t list[kSampleList], part[kFinishThreads / 64], start_mass[kBins];
  __shared__ uint32_t start[kBins];
  __shared__ uint64_t got[4];  // masses: top-k, top-p, min-p; the token's key
  __shared__ Digits digits;
  const int row = blockIdx.x, tid = threadIdx.x;
  const Row r = row_of(a, row);
  const uint64_t top = row_top<kFinishThreads>(a, row, part);
  const bool none = no_token(r, top);
  if (none || r.greedy) {
    if (tid == 0) {
      a.tokens[row] = none ? -1 : (int)key_index(top);
      if (a.logprobs) a.logprobs[row] = none ? __builtin_nanf("") : 0.f;
    }
    return;
  }
  const double zmax = (double)key_value(top);
  const double most = r.min_p > 0.f ? -log2((double)fminf(r.min_p, 1.f)) : 0.0;  // largest depth that min-p keeps
  uint32_t wanted;
  const Ends e = find_ends<kFinishThreads>(a, row, r, s, wanted);
  uint64_t total, token;
  if (wanted <= (uint32_t)kSampleList) {
    const int n = (int)wanted;
    int size = 64;
    while (size < n) size *= 2;
    for (int i = tid; i < size; i += kFinishThreads) list[i] = i < n ? row_list(a, row)[i] : 0;
    if (tid == 0) {
      got[0] = s.mass[e.kb + 1];
      got[1] = ~0ull;
      got[2] = e.mb >= 0 ? s.mass[e.mb] : ~0ull;
      got[3] = top;
    }
    // descending order
    for (int k = 2; k <= size; k *= 2)
      for (int j = k / 2; j > 0; j /= 2) {
        __syncthreads();
        for (int t = tid; t < size / 2; t += kFinishThreads) {
          const int i = 2 * t - (t & (j - 1)), o = i + j;
          const uint64_t x = list[i], y = list[o];
          if ((x < y) == ((i & k) == 0)) {
            list[i] = y;
            list[o] = x;
          }
        }
      }
    __syncthreads();
    // count and mass up to and with every element: its bin's start plus the
    // list's own prefix sums
    uint64_t w[kPer], sum = 0;
    int b[kPer];
    double d[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = tid * kPer + j;
      d[j] = i < n ? depth(zmax, key_value(list[i]), r.inv) : 0.0;
      b[j] = bin_of(d[j]);
      w[j] = i < n ? weight_of(d[j], a.unit) : 0;
      sum += w[j];
    }
    const uint64_t upto = wave_scan64(sum);
    if ((tid & 63) == 63) part[tid >> 6] = upto;
    __syncthreads();
    uint64_t before = upto - sum;
    for (int v = 0; v < (tid >> 6); ++v) before += part[v];
    uint64_t p = before;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = tid * kPer + j;
      if (i < n && (i == 0 || bin_of(depth(zmax, key_value(list[i - 1]), r.inv)) != b[j])) {
        start[b[j]] = (uint32_t)i;
        start_mass[b[j]] = p;
      }
      p += w[j];
    }
    __syncthreads();
    uint64_t m[kPer];
    p = before;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = tid * kPer + j;
      p += w[j];
      if (i >= n) continue;
      m[j] = s.mass[b[j]] + p - start_mass[b[j]];
      if (e.cut && b[j] == e.kb && s.count[b[j]] + i - start[b[j]] + 1 == r.k) got[0] = m[j];
      if (b[j] == e.mb && d[j] <= most) atomicMax(reinterpret_cast<unsigned long long*>(&got[2]), (unsigned long long)m[j]);
    }
    __syncthreads();
    if (e.p0 >= 0) {
      const double t = fmax((double)r.top_p * (double)got[0], 1.0);
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (tid * kPer + j < n && (double)(m[j] - w[j]) < t && (double)m[j] >= t) got[1] = m[j];
      __syncthreads();
    }
    total = min(min(got[0], got[1]), got[2]);
    const double t = (double)r.u * (double)total;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (tid * kPer + j < n && (double)(m[j] - w[j]) <= t && (double)m[j] > t) got[3] = list[tid * kPer + j];
    __syncthreads();
    token = got[3];
  } else {
    const auto* z = reinterpret_cast<const typename T::raw*>(a.logits) + (size_t)row * a.row_stride;
    total = s.mass[e.kb + 1];
    if (e.cut) total = search_row<T>(a, z, zmax, r, digits, [&](uint64_t c, uint64_t) { return c >= r.k; }).mass;
    uint64_t kept = total;
    if (e.p0 >= 0) {
      const double t = fmax((double)r.top_p * (double)total, 1.0);
      kept = search_row<T>(a, z, zmax, r, digits, [&](uint64_t, uint64_t m) { return (double)m >= t; }).mass;
    }
    if (e.mb >= 0) {
      uint64_t sum = 0;
      each8<T, kFinishThreads>(z, 0, a.vocab, [&](const float(&v)[8], int, int n) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const double d = depth(zmax, v[j], r.inv);
          if (j < n && d <= most) sum += weight_of(d, a.unit);
        }
      });
      sum = wave_sum64(sum);
      if ((tid & 63) == 0) part[tid >> 6] = sum;
      __syncthreads();
      sum = 0;
      for (int v = 0; v < kFinishThreads / 64; ++v) sum += part[v];
      kept = min(kept, sum);
      __syncthreads();
    }
    total = min(total, kept);
    const double t = (double)r.u * (double)total;
    token = search_row<T>(a, z, zmax, r, digits, [&](uint64_t, uint64_t m) { return (double)m > t; }).key;
  }
  if (tid == 0) {
    a.tokens[row] = (int)key_index(token);
    // log of the weight over the kept total, both relative to the largest weight
    if (a.logprobs)
      a.logprobs[row] = (float)(-0.6931471805599453 * depth(zmax, key_value(token), r.inv) - log(ldexp((double)total, -a.unit)));
  }
}

template <class T>
int launch_type(const SampleArgs& a, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  const dim3 chunks(a.batch * a.nchunk);
  hipLaunchKernelGGL(sample_max_kernel<T>, chunks, dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(sample_bins_kernel<T>, chunks, dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(sample_gather_kernel<T>, chunks, dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(sample_finish_kernel<T>, dim3(a.batch), dim3(kFinishThreads), 0, st, a);
  return (int)hipGetLastError();
}

}  // namespace

int launch_sample(const SampleArgs& a, int type, void* stream) {
  switch (type) {
    case 0: return launch_type<F32>(a, stream);
    case 1: return launch_type<F16>(a, stream);
    case 2: return launch_type<BF16>(a, stream);
    default: return (int)hipErrorInvalidValue;
  }
}

}  // namespace kvq
