// The next token of every row of logits (gfx950): temperature, top-k, top-p and
// min-p, one given uniform number per row (include/dgap.h states the rule).
//
// All filters keep a prefix of the row's descending order (equal logits by
// lower index), and the token is the element at which the kept mass, summed in
// that order, passes u times the kept total: every step is a search for the
// element where a count or a mass reaches a target.  With d = log2(e) / T
// (z_max - z) an element weighs 2^-d.
//   max     the row's largest logit
//   bins    counts and masses of 2048 bins of d, 1/40 of an octave each
//   ends    from the bins' prefix sums the bins where the searches end (a
//           bracket of bins, where a target depends on an earlier search)
//   select  the elements of those bins, a few hundred, listed; the
//           searches ended among them, a digit of the keys at a time
// Few rows: max and bins take one workgroup per (row, chunk), ends and select
// one per row (three launches).  Many rows: one workgroup per row takes all
// steps, reading the row three times (the second and third time from cache).
//
// A weight is a 24-bit number M 2^-n (n = floor(d), one hardware exponential of
// the rest, d itself in 64 bits), and all elements of a bin share n, so a bin's
// mass is a whole number, counted up with its elements in one 64-bit atomic;
// masses across bins are whole numbers of 2^-unit of the largest weight (unit is
// 45, 38 for the largest vocabularies): a sum of M is rounded down to them, never
// an M alone, or the elements of deep bins would add up to less than the bin.  Sums
// are exact: they depend neither on the order of the atomics nor on whether a
// bin, the list or a search over the row summed an element.  Elements of the last
// bin, 51 octaves down, count as 0 and are never chosen.  Where the bins that the
// searches end in hold more elements than a list (thousands of equal logits), each
// search goes over all the row's logits, a digit of the keys at a time.
//
// What bounds it: latency, along one workgroup's dependent steps: of one row's 24
// us (128256 fp32, top-k 50 and top-p 0.95, an input whose three searches all go by
// digits; 19 to 21 over many inputs) max 3 and bins 5, then the ends 3.5,
// listing 6 (the compares, at four waves per SIMD: with every load asked for at
// once it takes as long) and the three searches 4, one step after the other.  Many
// rows: 256 flat ones of 128256 fp16 60 us, of which 11 go to the first read (all
// that comes from HBM, 13 at a copy's rate), 21 to the bins, about twenty
// instructions a logit (without their atomics, with the chains of a load side by
// side, or in fixed point, 20 to 21), and 27 to listing and searching.  Sorting the
// list took 5 to 22 us where the digit searches take 4 to 8; straight-line code for
// every match of a load, run once from a cold instruction cache, cost more than a
// loop.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "decode_common.h"
#include "kvq_internal.h"
#include "logits_common.h"

namespace kvq {
namespace {

using namespace logits;

constexpr int kThreads = 256;
constexpr int kRowThreads = 1024;
constexpr int kAhead = 4;  // loads under way of a thread of those as it lists elements
constexpr int kGroup = kSampleGroup;
static_assert(kGroup == 64 * 8, "a wave's loads");
constexpr int kBins = kSampleBins;
constexpr int kPerOctave = 40;  // 51 octaves: past them no weight is left (unit <= 45)
// a bin while its elements are counted: their number above bit kCount, the sum
// of their M below (of a chunk or a row of up to 2^19: 2^43)
constexpr int kCount = 44;
constexpr uint64_t kSum = (1ull << kCount) - 1;

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

// An element's bin and M.
struct Place {
  int bin;
  uint32_t m;
};
__device__ __forceinline__ Place place_of(double d) {
  d = fmin(d, 60.0);
  const int n = (int)d;
  const float f = fminf((float)__builtin_amdgcn_fract(d), 0x1.fffffep-1f);
  return {min(n * kPerOctave + (int)(f * (float)kPerOctave), kBins - 1),
          (uint32_t)(__builtin_amdgcn_exp2f(-f) * 16777216.f)};
}
// M or a sum of them in a bin, in units of 2^-unit
__device__ __forceinline__ uint64_t mass_of(uint64_t m, int bin, int unit) {
  const int sh = unit - 24 - bin / kPerOctave;
  return sh >= 0 ? m << sh : m >> -sh;
}

__device__ __forceinline__ uint64_t* row_bins(const SampleArgs& a, int row) {
  return reinterpret_cast<uint64_t*>(a.ws + (size_t)row * a.row_bytes);
}
// (vocabularies past 2^19 count their bins' elements apart)
__device__ __forceinline__ uint32_t* row_count(const SampleArgs& a, int row) {
  return reinterpret_cast<uint32_t*>(row_bins(a, row) + kBins);
}
// the groups' largest logits, then the chunks'
__device__ __forceinline__ float* row_groups(const SampleArgs& a, int row) {
  return reinterpret_cast<float*>(row_count(a, row) + kBins);
}
__device__ __forceinline__ float* row_top(const SampleArgs& a, int row) { return row_groups(a, row) + a.ngroup; }
template <class T>
__device__ __forceinline__ const typename T::raw* row_logits(const SampleArgs& a, int row) {
  return reinterpret_cast<const typename T::raw*>(a.logits) + (size_t)row * a.row_stride;
}

// 8 logits from i on, or the last 8 of those below bulk (>= 8): loads without a
// branch around them, which would end the overlap of several.
template <class T>
__device__ __forceinline__ raw8_t<T> load_below(const typename T::raw* z, int i, int bulk) {
  return load8<T>(z + min(i, bulk - 8));
}

// f(logit, index) for the logits [from, to), 8 a thread at a time with the next
// load on its way, then the last few one by one.
template <class T, int NT, class F>
__device__ __forceinline__ void each(const typename T::raw* z, int from, int to, F f) {
  const int bulk = from + ((to - from) & ~7);
  int i = from + 8 * (int)threadIdx.x;
  if (bulk > from) {
    raw8_t<T> v = load_below<T>(z, i, bulk);
#pragma unroll 1
    for (; i < bulk; i += 8 * NT) {
      const raw8_t<T> x = v;
      v = load_below<T>(z, i + 8 * NT, bulk);
#pragma unroll
      for (int j = 0; j < 8; ++j) f(T::value(x[j]), i + j);
    }
  }
  i = bulk + (int)threadIdx.x;
  if (i < to) f(T::value(z[i]), i);
}

// The largest of the logits [from, to), in every thread; +inf where one is NaN
// or +inf.  from is a multiple of kGroup; groups: the row's, one per kGroup
// logits, of which this writes its own (a wave's loads at a time).
template <class T, int NT>
__device__ __forceinline__ float top_of(const typename T::raw* z, int from, int to, float* groups, float* part) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, bulk = from + ((to - from) & ~7);
  float top = -__builtin_inff();
  bool bad = false;
  constexpr int U = NT == kRowThreads ? 4 : 1;  // (a row's one workgroup: four loads under way)
  for (int g = from + kGroup * wv; g < to; g += 8 * NT * U) {
    raw8_t<T> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (bulk > from) v[u] = load_below<T>(z, g + 8 * NT * u + 8 * lane, bulk);
      else v[u] = all8<T>(-__builtin_inff());
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int g0 = g + 8 * NT * u;
      float m = -__builtin_inff();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // (past the end the last 8 again, which the group's maximum may hold: they
        // are below bulk, and a group's maximum is a bound)
        const float x = T::value(v[u][j]);
        m = fmaxf(m, x);
        bad |= !(x < __builtin_inff());
      }
      if (g0 + kGroup > bulk && g0 < to && bulk + lane < to) {  // the last few, of the last group
        const float x = T::value(z[bulk + lane]);
        m = fmaxf(m, x);
        bad |= !(x < __builtin_inff());
      }
      m = dec::wave_max(m);
      if (lane == 0 && g0 < to) groups[g0 / kGroup] = m;
      top = fmaxf(top, m);
    }
  }
  if (__builtin_amdgcn_ballot_w64(bad)) top = __builtin_inff();
  if (lane == 0) part[wv] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) top = fmaxf(top, part[w]);
  return top;
}

// Counts the logits [from, to) into bins (LDS, cleared).
template <class T, int NT>
__device__ __forceinline__ void count_bins(const typename T::raw* z, int from, int to, double zmax, double inv, uint64_t* bins) {
  uint32_t rest = 0;  // elements of the last bin: their mass is 0
  each<T, NT>(z, from, to, [&](float x, int) {
    const Place p = place_of(depth(zmax, x, inv));
    if (p.bin == kBins - 1)
      ++rest;
    else
      atomicAdd(reinterpret_cast<unsigned long long*>(&bins[p.bin]), (1ull << kCount) | p.m);
  });
  if (rest) atomicAdd(reinterpret_cast<unsigned long long*>(&bins[kBins - 1]), (unsigned long long)rest << kCount);
}

template <class T>
__global__ __launch_bounds__(kThreads) void sample_max_kernel(SampleArgs a) {
  __shared__ float part[kThreads / 64];
  const int row = blockIdx.x / a.nchunk, chunk = blockIdx.x % a.nchunk, tid = threadIdx.x;
  // this workgroup's share of the row's bins starts at 0
  const int share = (kBins + a.nchunk - 1) / a.nchunk;
  for (int b = chunk * share + tid; b < min(kBins, (chunk + 1) * share); b += kThreads) {
    row_bins(a, row)[b] = 0;
    row_count(a, row)[b] = 0;
  }
  const int from = chunk * a.chunk, to = min(a.vocab, from + a.chunk);
  const float m = top_of<T, kThreads>(row_logits<T>(a, row), from, to, row_groups(a, row), part);
  if (tid == 0) row_top(a, row)[chunk] = m;
}

// The row's largest logit from its chunks', in every thread.
template <int NT>
__device__ __forceinline__ float join_top(const SampleArgs& a, int row, float* part) {
  float m = -__builtin_inff();
  for (int c = threadIdx.x; c < a.nchunk; c += NT) m = fmaxf(m, row_top(a, row)[c]);
  m = dec::wave_max(m);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) m = fmaxf(m, part[w]);
  return m;
}
// A row without a token to sample: settings out of range, NaN or +inf, nothing finite.
__device__ __forceinline__ bool no_token(const Row& r, float top) { return r.bad || not_finite(top); }

template <class T>
__global__ __launch_bounds__(kThreads) void sample_bins_kernel(SampleArgs a) {
  __shared__ uint64_t bins[kBins];
  __shared__ float part[kThreads / 64];
  const int row = blockIdx.x / a.nchunk, chunk = blockIdx.x % a.nchunk, tid = threadIdx.x;
  const Row r = row_of(a, row);
  if (r.bad || r.greedy) return;
  for (int b = tid; b < kBins; b += kThreads) bins[b] = 0;
  const float top = join_top<kThreads>(a, row, part);
  if (no_token(r, top)) return;
  const int from = chunk * a.chunk, to = min(a.vocab, from + a.chunk);
  count_bins<T, kThreads>(row_logits<T>(a, row), from, to, (double)top, r.inv, bins);
  __syncthreads();
  const bool wide = a.vocab > kSampleNarrow;
  for (int b = tid; b < kBins; b += kThreads) {
    const uint64_t x = bins[b];
    if (x == 0) continue;
    if (wide) atomicAdd(&row_count(a, row)[b], (uint32_t)(x >> kCount));
    atomicAdd(reinterpret_cast<unsigned long long*>(&row_bins(a, row)[b]), (unsigned long long)(wide ? x & kSum : x));
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
  uint64_t part[kRowThreads / 64][2];
  int found[6];
};

// A thread's bins (kPer * tid on): their counts and sums of M.
constexpr int kPer = kBins / kRowThreads;
struct OwnBins {
  uint32_t count[kPer];
  uint64_t sum[kPer];
};

__device__ __forceinline__ Ends find_ends(const SampleArgs& a, const Row& r, Prefix& s, uint32_t& wanted, const OwnBins& own) {
  constexpr int NT = kRowThreads;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  uint64_t m[kPer], msum = 0;
  uint32_t csum = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    m[j] = mass_of(own.sum[j], tid * kPer + j, a.unit);
    msum += m[j];
    csum += own.count[j];
  }
  const uint64_t mi = wave_scan64(msum), ci = wave_scan64(csum);
  if (lane == 63) {
    s.part[wv][0] = mi;
    s.part[wv][1] = ci;
  }
  if (tid < 6) s.found[tid] = -1;
  __syncthreads();
  uint64_t mass[kPer + 1], mb = mi - msum, cb = ci - csum;
  uint32_t count[kPer + 1];
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const uint64_t x = s.part[w][0], y = s.part[w][1];
    mb += w < wv ? x : 0;
    cb += w < wv ? y : 0;
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    s.mass[tid * kPer + j] = mass[j] = mb;
    s.count[tid * kPer + j] = count[j] = (uint32_t)cb;
    mb += m[j];
    cb += own.count[j];
  }
  mass[kPer] = mb;
  count[kPer] = (uint32_t)cb;
  if (tid == NT - 1) {
    s.mass[kBins] = mb;
    s.count[kBins] = (uint32_t)cb;
  }
  // the bin in which a test becomes true (of the count and mass before it, then with it)
  auto search = [&](int slot, auto test) {
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (!test(count[j], mass[j]) && test(count[j + 1], mass[j + 1])) s.found[slot] = tid * kPer + j;
  };
  Ends e;
  search(0, [&](uint32_t n, uint64_t) { return n >= r.k; });
  __syncthreads();
  e.kb = s.found[0];
  // (the last bin has no mass: it is never cut)
  e.cut = e.kb < kBins - 1 && s.count[e.kb + 1] != r.k;
  const double lo = (double)(e.cut ? s.mass[e.kb] : s.mass[e.kb + 1]), hi = (double)s.mass[e.kb + 1];
  e.p0 = e.p1 = -1;
  if (r.top_p < 1.f) {
    const double t0 = fmax((double)r.top_p * lo, 1.0), t1 = fmax((double)r.top_p * hi, 1.0);
    search(1, [&](uint32_t, uint64_t w) { return (double)w >= t0; });
    search(2, [&](uint32_t, uint64_t w) { return (double)w >= t1; });
    __syncthreads();
    e.p0 = s.found[1];
    e.p1 = s.found[2];
  }
  e.mb = -1;
  if (r.min_p > 0.f && r.min_p <= 1.f) {
    e.mb = place_of(-log2((double)r.min_p)).bin;
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
  // what lies past the end decides nothing
  if (e.p0 > end1) e.p0 = e.p1 = -1;
  e.p1 = min(e.p1, end1);
  if (e.mb > end1) e.mb = -1;
  if (e.kb > end1 && e.p0 < 0) e.cut = false;
  const double t0 = (double)r.u * (double)s.mass[end0], t1 = (double)r.u * (double)s.mass[end1 + 1];
  search(3, [&](uint32_t, uint64_t w) { return (double)w > t0; });
  search(4, [&](uint32_t, uint64_t w) { return (double)w > t1; });
  __syncthreads();
  e.u0 = s.found[3];
  e.u1 = s.found[4];
  uint32_t held = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    if (e.wanted(tid * kPer + j)) held += own.count[j];
  const uint64_t all = wave_sum64(held);
  if (lane == 0) s.part[wv][0] = all;
  __syncthreads();
  wanted = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) wanted += (uint32_t)s.part[w][0];
  return e;
}

// A search over a row's elements of one bin that are not listed, a digit of the
// keys at a time: the first element, in descending order, with which past(their
// count, their sum of M) holds; mass: the M up to and with it.
struct Found {
  uint64_t key, mass;
};
struct Digits {
  uint64_t mass[256];
  uint32_t count[256];
  uint64_t before[2];
  uint32_t digit;
};
template <class T, class F>
__device__ __forceinline__ Found search_row(const SampleArgs& a, const typename T::raw* z, double zmax, const Row& r, int bin, Digits& s, F past) {
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
#pragma unroll 1
    for (int base = 0; base < a.vocab; base += kRowThreads) {  // (every lane stays: waves add up together)
      const int i = base + (int)threadIdx.x;
      const float value = i < a.vocab ? T::value(z[i]) : -__builtin_inff();
      const uint64_t key = make_key(value, i);
      bool in = i < a.vocab && (shift == 56 || (key >> (shift + 8)) == prefix);
      if (!__builtin_amdgcn_ballot_w64(in)) continue;
      const Place p = place_of(depth(zmax, value, r.inv));
      in = in && p.bin == bin;
      const uint64_t some = __builtin_amdgcn_ballot_w64(in);
      if (!some) continue;
      const uint64_t w = in ? p.m : 0;
      const uint32_t digit = (uint32_t)(key >> shift) & 255u;
      const uint32_t common = (uint32_t)__builtin_amdgcn_readlane((int)digit, __builtin_ctzll(some));
      if (__builtin_amdgcn_ballot_w64(in && digit != common) == 0) {
        const uint64_t all = wave_sum64(w);
        if ((threadIdx.x & 63) == 0) {
          atomicAdd(&s.count[common], (uint32_t)__builtin_popcountll(some));
          atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[common]), (unsigned long long)all);
        }
      } else if (in) {
        atomicAdd(&s.count[digit], 1u);
        atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[digit]), (unsigned long long)w);
      }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      // (rounding may have moved the target past the end: then the last element)
      uint64_t n = count, m = mass;
      for (int d = 255; d >= 0; --d) {
        if (s.count[d] == 0) continue;
        s.digit = (uint32_t)d;
        s.before[0] = n;
        s.before[1] = m;
        n += s.count[d];
        m += s.mass[d];
        if (past((uint32_t)n, m)) break;
      }
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

// Logits that hold those of the bins b0 .. b1, a hundredth of a bin wider, and
// a step of fp32 at either end.  step: logits per bin.
struct Range {
  float lo, hi;
  // (two instructions; none: +inf to +inf, which no listed logit is)
  __device__ __forceinline__ bool has(float v) const { return __builtin_amdgcn_fmed3f(v, lo, hi) == v; }
};
__device__ __forceinline__ float step_from(float f, int by) {  // to the next float down (-1) or up (1)
  const int i = __builtin_bit_cast(int, f);
  if (f == 0.f) return __builtin_bit_cast(float, by < 0 ? (int)0x80000001 : 1);
  if (not_finite(f)) return f;
  return __builtin_bit_cast(float, i + (i < 0 ? -by : by));
}
__device__ __forceinline__ Range range_of(double zmax, double step, int b0, int b1) {
  if (b1 < b0) return {__builtin_inff(), __builtin_inff()};
  return {step_from((float)(zmax - ((double)b1 + 1.01) * step), -1), step_from((float)(zmax - ((double)b0 - 0.01) * step), 1)};
}

constexpr int kListPer = kSampleList / kRowThreads;
struct Select {
  Prefix s;
  union {
    uint64_t bins[kBins];  // until the prefix sums are taken
    uint2 list[kSampleList];  // logit, index
    Digits digits;
  };
  uint64_t part[kRowThreads / 64];
  uint64_t digit[3][256];  // of a search in the list: counts above bit kCount, sums of M below
  uint64_t found[2];
  uint32_t held;
  float top[kRowThreads / 64];
};

__device__ __forceinline__ void put_token(const SampleArgs& a, int row, int token, float logprob) {
  if (threadIdx.x != 0) return;
  a.tokens[row] = token;
  if (a.logprobs) a.logprobs[row] = logprob;
}

// Rows that need no search: no token, or the largest logit.  False for the others.
template <class T>
__device__ __forceinline__ bool simple_row(const SampleArgs& a, int row, const Row& r, float top, const float* groups, Select& m) {
  if (no_token(r, top)) {
    put_token(a, row, -1, __builtin_nanf(""));
    return true;
  }
  if (!r.greedy) return false;
  if (threadIdx.x == 0) m.held = ~0u;
  __syncthreads();
  uint32_t first = ~0u;
  for (int g = threadIdx.x >> 6; g < a.ngroup; g += kRowThreads / 64) {
    if (groups[g] != top) continue;
    for (int i = kGroup * g + (threadIdx.x & 63); i < min(a.vocab, kGroup * (g + 1)); i += 64)
      if (T::value(row_logits<T>(a, row)[i]) == top) first = min(first, (uint32_t)i);
  }
  if (first != ~0u) atomicMin(&m.held, first);
  __syncthreads();
  put_token(a, row, (int)m.held, 0.f);
  return true;
}

// The sum over the workgroup, in every thread.
__device__ __forceinline__ uint64_t block_sum(uint64_t v, uint64_t* part) {
  v = wave_sum64(v);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int w = 0; w < kRowThreads / 64; ++w) v += part[w];
  __syncthreads();
  return v;
}

// The list's element that a thread holds: its key in as few bits as its type
// and the vocabulary need (value above index_bits, the index's complement below).
struct Held {
  uint64_t key;
  int bin;      // -1: none, or not of a wanted bin
  uint32_t m;
  bool near;    // min-p keeps it
};
template <class T>
__device__ __forceinline__ uint64_t short_key(uint32_t order, uint32_t index, int index_bits) {
  return ((uint64_t)(order >> T::kZeroBits) << index_bits) | (~index & ((1u << index_bits) - 1u));
}

// In the list's elements of one bin, in descending order, the first with which
// past(their count, their sum of M) holds; mass: the M up to and with it.  range:
// of the bin's logits, whose keys share the bits above the first digit; alone:
// the bin has one element.  digits
// all zero on entry and exit; one barrier a digit: a digit's counts go to one of
// three arrays, the next one's is cleared meanwhile.
template <class T, class F>
__device__ __forceinline__ Found search_bin(const Held (&c)[kListPer], int bin, const Range& range, int index_bits,
                                            bool alone, uint64_t (&digits)[3][256], uint64_t (&found)[2], F past) {
  const int tid = threadIdx.x, lane = tid & 63;
  if (alone) {  // whoever holds it says so
#pragma unroll
    for (int j = 0; j < kListPer; ++j)
      if (c[j].bin == bin) {
        found[0] = c[j].key;
        found[1] = c[j].m;
      }
    __syncthreads();
    const Found f = {found[0], found[1]};
    __syncthreads();
    return f;
  }
  const uint64_t hi = short_key<T>(order_bits(range.hi), 0u, index_bits), lo = short_key<T>(order_bits(range.lo), ~0u, index_bits);
  int top = hi == lo ? 1 : 64 - __builtin_clzll(hi ^ lo);  // bits that may differ
  uint64_t prefix = hi >> top, before = 0;                 // before: count and sum above the prefix
  for (int turn = 0;; turn = turn == 2 ? 0 : turn + 1) {
    const int width = min(8, top), shift = top - width;
#pragma unroll
    for (int j = 0; j < kListPer; ++j)
      if (c[j].bin == bin && (c[j].key >> top) == prefix)
        atomicAdd(reinterpret_cast<unsigned long long*>(&digits[turn][(c[j].key >> shift) & ((1u << width) - 1u)]),
                  (1ull << kCount) | c[j].m);
    if (tid < 256) digits[turn == 2 ? 0 : turn + 1][tid] = 0;
    __syncthreads();
    // lane l: digits 255 - 4 l down to 252 - 4 l
    uint64_t own[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      own[j] = digits[turn][255 - 4 * lane - j];
      sum += own[j];
    }
    uint64_t upto = before + wave_scan64(sum) - sum, at = 0, in = 0;
    uint32_t digit = 256;
    // (rounding may have moved the target past the end: then the last element)
    uint64_t last_at = 0, last_in = 0;
    uint32_t last = 256;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t next = upto + own[j];
      if (own[j] != 0) {
        last = 255 - 4 * lane - j;
        last_at = upto;
        last_in = own[j];
        if (digit == 256 && past((uint32_t)(next >> kCount), next & kSum)) {
          digit = last;
          at = upto;
          in = own[j];
        }
      }
      upto = next;
    }
    const uint64_t who = __builtin_amdgcn_ballot_w64(digit != 256), some = __builtin_amdgcn_ballot_w64(last != 256);
    const int w = who ? __builtin_ctzll(who) : some ? 63 - __builtin_clzll(some) : 0;
    before = lane64(who ? at : last_at, w);
    in = lane64(who ? in : last_in, w);
    prefix = (prefix << width) | (uint32_t)__builtin_amdgcn_readlane((int)(who ? digit : last), w);
    top = shift;
    if (top > 0 && in >> kCount > 1) continue;
    // the one element left: whoever holds it says so
    __syncthreads();  // (every wave has read the digits)
    if (tid < 256) digits[0][tid] = digits[1][tid] = digits[2][tid] = 0;
#pragma unroll
    for (int j = 0; j < kListPer; ++j)
      if (c[j].bin == bin && (c[j].key >> top) == prefix) found[0] = c[j].key;
    __syncthreads();
    const uint64_t key = found[0];
    return {key, (before + in) & kSum};
  }
}

// The group that a lane looks at, of those from g0 on.
__device__ __forceinline__ int own_group(int g0) {
  return g0 + (kRowThreads / 64) * (threadIdx.x & 63) + (threadIdx.x >> 6);
}

// The row's token once its bins' prefix sums and ends are known.  groups: the
// largest logit of every kGroup ones; first: of own_group(0).
template <class T>
__device__ __forceinline__ void select(const SampleArgs& a, int row, const Row& r, float top, const float* groups,
                                       float first, const Ends& e, uint32_t wanted, Select& m) {
  Prefix& s = m.s;
  const int tid = threadIdx.x;
  const double zmax = (double)top;
  const double most = r.min_p > 0.f ? -log2((double)fminf(r.min_p, 1.f)) : 0.0;  // largest depth that min-p keeps
  const auto* z = row_logits<T>(a, row);
  const double step = 1.0 / (kPerOctave * r.inv);
  const bool listed = wanted <= (uint32_t)kSampleList;
  const int index_bits = 32 - __builtin_clz((uint32_t)a.vocab);
  Held c[kListPer];
#pragma unroll
  for (int j = 0; j < kListPer; ++j) c[j] = {0, -1, 0, false};
  if (listed) {
    if (tid == 0) m.held = 0;
    if (tid < 256) m.digit[0][tid] = m.digit[1][tid] = m.digit[2][tid] = 0;
    __syncthreads();
    // the filters' bins, and the token's
    int b0 = kBins, b1 = -1;
    for (int b : {e.cut ? e.kb : -1, e.p0, e.p1, e.mb})
      if (b >= 0) {
        b0 = min(b0, b);
        b1 = max(b1, b);
      }
    const Range x = range_of(zmax, step, e.u0, e.u1), y = range_of(zmax, step, b0, b1);
    const float least = fminf(x.lo, y.lo);
    const int wv = tid >> 6, lane = tid & 63, bulk = a.vocab & ~7;
    auto list = [&](auto sift_c) __attribute__((always_inline)) {
      auto put = [&](float value, int i) {
        if (decltype(sift_c)::value && !e.wanted(place_of(depth(zmax, value, r.inv)).bin)) return;
        const uint32_t slot = atomicAdd(&m.held, 1u);
        if (slot < (uint32_t)kSampleList) m.list[slot] = make_uint2(__builtin_bit_cast(uint32_t, value), (uint32_t)i);
      };
      for (int g0 = 0; bulk > 0 && g0 < a.ngroup; g0 += kRowThreads) {
        // groups g0 + 16 l + wv that reach the wanted bins
        const int own = own_group(g0);
        const float held = g0 > 0 ? groups[min(own, a.ngroup - 1)] : first;
        uint64_t left = __builtin_amdgcn_ballot_w64(own < a.ngroup && held >= least);
        int group[kAhead];  // -1: none left
        raw8_t<T> v[kAhead];
        auto next = [&](int u) {
          group[u] = left ? g0 + (kRowThreads / 64) * __builtin_ctzll(left) + wv : -1;
          left &= left - 1;
          v[u] = load_below<T>(z, kGroup * max(group[u], 0) + 8 * lane, bulk);
        };
#pragma unroll
        for (int u = 0; u < kAhead; ++u) next(u);
        while (group[0] >= 0) {
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            if (group[u] < 0) break;
            const int at = kGroup * group[u] + 8 * lane;
            uint32_t hits = 0;  // (no branch per logit)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float value = T::value(v[u][j]);
              hits |= x.has(value) | y.has(value) ? 1u << j : 0u;
            }
            hits = at < bulk ? hits : 0u;
#pragma unroll 1
            while (hits) {
              const int j = __builtin_ctz(hits);
              hits &= hits - 1;
              float value = T::value(v[u][0]);
#pragma unroll
              for (int o = 1; o < 8; ++o) value = j == o ? T::value(v[u][o]) : value;
              put(value, at + j);
            }
            next(u);
          }
        }
      }
      if (bulk + tid < a.vocab) {
        const float value = T::value(z[bulk + tid]);
        if (x.has(value) || y.has(value)) put(value, bulk + tid);
      }
    };
    // Between the filters' bins others may lie (top-k's thousands below the end of
    // top-p), and a range's end, rounded outwards to fp32, may be bins away: where
    // that is more than the list takes, every hit's bin is looked at before it is put.
    bool sift = b1 > b0 && s.count[b1 + 1] - s.count[b0] > (uint32_t)kSampleList;
    if (!sift) {
      list(std::false_type{});
      __syncthreads();
      sift = m.held > (uint32_t)kSampleList;
      if (sift) {
        __syncthreads();
        if (tid == 0) m.held = 0;
        __syncthreads();
      }
    }
    if (sift) list(std::true_type{});
    __syncthreads();
    const int n = (int)m.held;
#pragma unroll
    for (int j = 0; j < kListPer; ++j) {
      const int i = kRowThreads * j + tid;
      if (kRowThreads * j >= n) continue;
      const uint2 x = i < n ? m.list[i] : make_uint2(0, 0);
      const float value = __builtin_bit_cast(float, x.x);
      const double d = depth(zmax, value, r.inv);
      const Place p = place_of(d);
      c[j].key = short_key<T>(order_bits(value + 0.f), x.y, index_bits);
      c[j].bin = i < n && e.wanted(p.bin) ? p.bin : -1;
      c[j].m = p.m;
      c[j].near = d <= most;
    }
    __syncthreads();
  }
  // one search after the other: top-k, top-p, (min-p), the token; in the list,
  // in the bin that the target lies in, or over the whole row
  uint64_t total = s.mass[e.kb + 1], kept = ~0ull, token = 0;
#pragma unroll 1
  for (int turn = e.cut ? 0 : e.p0 >= 0 ? 1 : 2; turn < 3; ++turn) {
    if (turn == 1 && e.p0 < 0) continue;
    if (turn == 2) {
      if (e.mb >= 0) {
        uint64_t sum = 0;
        if (listed) {
#pragma unroll
          for (int j = 0; j < kListPer; ++j)
            if (c[j].bin == e.mb && c[j].near) sum += c[j].m;
        } else {
          each<T, kRowThreads>(z, 0, a.vocab, [&](float value, int) {
            const double d = depth(zmax, value, r.inv);
            const Place p = place_of(d);
            if (p.bin == e.mb && d <= most) sum += p.m;
          });
        }
        sum = mass_of(block_sum(sum, m.part), e.mb, a.unit) + s.mass[e.mb];
        kept = min(kept, sum);
      }
      total = min(total, kept);
    }
    const double t = turn == 1 ? fmax((double)r.top_p * (double)total, 1.0) : (double)r.u * (double)total;
    auto past = [&](uint32_t count, uint64_t mass) {
      return turn == 0 ? count >= r.k : turn == 1 ? (double)mass >= t : (double)mass > t;
    };
    int b = turn == 0 ? e.kb : turn == 1 ? e.p0 : e.u0;
    const int last = turn == 0 ? e.kb : turn == 1 ? e.p1 : e.u1;
    while (b < last && !past(s.count[b + 1], s.mass[b + 1])) ++b;
    const uint64_t base = s.mass[b];
    const uint32_t before = s.count[b];
    auto past_in = [&](uint32_t count, uint64_t sum) { return past(before + count, base + mass_of(sum, b, a.unit)); };
    Found f;
    if (listed)
      f = search_bin<T>(c, b, range_of(zmax, step, b, b), index_bits, s.count[b + 1] - before == 1, m.digit, m.found, past_in);
    else
      f = search_row<T>(a, z, zmax, r, b, m.digits, past_in);
    f.mass = base + mass_of(f.mass, b, a.unit);
    if (turn == 0) total = f.mass;
    if (turn == 1) kept = f.mass;
    token = f.key;
  }
  if (listed) {
    // back to a whole key (the dropped bits of a negative value's are ones)
    const uint32_t order = (uint32_t)(token >> index_bits) << T::kZeroBits;
    token = ((uint64_t)(order & 0x80000000u ? order : order | ((1u << T::kZeroBits) - 1u)) << 32) |
            (uint32_t)(token | (~0u << index_bits));
  }
  // log of the weight over the kept total, both relative to the largest weight
  put_token(a, row, (int)key_index(token),
            (float)(-0.6931471805599453 * depth(zmax, key_value(token), r.inv) - log(ldexp((double)total, -a.unit))));
}

template <class T>
__global__ __launch_bounds__(kRowThreads) void sample_finish_kernel(SampleArgs a) {
  __shared__ Select m;
  const int row = blockIdx.x;
  // what later steps read is under way from the start (greedy rows: contents undefined, unused)
  const bool wide = a.vocab > kSampleNarrow;
  const float* groups = row_groups(a, row);
  const float first = groups[min(own_group(0), a.ngroup - 1)];
  OwnBins own;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const uint64_t x = row_bins(a, row)[threadIdx.x * kPer + j];
    const uint32_t n = row_count(a, row)[threadIdx.x * kPer + j];
    own.count[j] = wide ? n : (uint32_t)(x >> kCount);
    own.sum[j] = wide ? x : x & kSum;
  }
  const Row r = row_of(a, row);
  const float top = join_top<kRowThreads>(a, row, m.top);
  if (simple_row<T>(a, row, r, top, groups, m)) return;
  uint32_t wanted;
  const Ends e = find_ends(a, r, m.s, wanted, own);
  select<T>(a, row, r, top, groups, first, e, wanted, m);
}

template <class T>
__global__ __launch_bounds__(kRowThreads) void sample_row_kernel(SampleArgs a) {
  __shared__ Select m;
  __shared__ float groups[kSampleNarrow / kGroup];
  const int row = blockIdx.x;
  const Row r = row_of(a, row);
  for (int b = threadIdx.x; b < kBins; b += kRowThreads) m.bins[b] = 0;
  const float top = top_of<T, kRowThreads>(row_logits<T>(a, row), 0, a.vocab, groups, m.top);
  if (simple_row<T>(a, row, r, top, groups, m)) return;
  count_bins<T, kRowThreads>(row_logits<T>(a, row), 0, a.vocab, (double)top, r.inv, m.bins);
  __syncthreads();
  OwnBins own;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const uint64_t x = m.bins[threadIdx.x * kPer + j];
    own.count[j] = (uint32_t)(x >> kCount);
    own.sum[j] = x & kSum;
  }
  uint32_t wanted;
  const Ends e = find_ends(a, r, m.s, wanted, own);
  select<T>(a, row, r, top, groups, groups[min(own_group(0), a.ngroup - 1)], e, wanted, m);
}

template <class T>
int launch_type(const SampleArgs& a, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  if (a.nchunk == 0) {
    hipLaunchKernelGGL(sample_row_kernel<T>, dim3(a.batch), dim3(kRowThreads), 0, st, a);
    return (int)hipGetLastError();
  }
  const dim3 chunks(a.batch * a.nchunk);
  hipLaunchKernelGGL(sample_max_kernel<T>, chunks, dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(sample_bins_kernel<T>, chunks, dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(sample_finish_kernel<T>, dim3(a.batch), dim3(kRowThreads), 0, st, a);
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
