// Host side of the block-scaled caches (include/kvq.h): descriptors, the split plan
// of their attention, and its launches.  Lengths, pages and appends are the packed
// caches' (kvq_api.cpp).
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "kvq.h"
#include "kvq_host.h"
#include "kvq_internal.h"

using kvq::fail;

namespace {

// Rows of an attention launch: nqry queries per sequence in row groups of qpr
// queries (DecodeArgs).
struct Rows {
  int nqry = 1, qpr = 1, nrg = 1, rows = 16;
};

Rows rows_for(const kvq_cache* c, int nqry) {
  const int gqh = c->d.num_q_heads / c->d.num_kv_heads;
  Rows r;
  r.nqry = nqry;
  r.qpr = std::min(nqry, r.rows / gqh);
  r.nrg = (nqry + r.qpr - 1) / r.qpr;
  return r;
}

// Workgroups per sequence and split.
int64_t units_of(const kvq_cache* c, const Rows& r) { return (int64_t)c->d.num_kv_heads * r.nrg; }

// Workgroups that a call is split into at most (its records, which the workspace
// holds at any lengths, grow with them).
int64_t most_workgroups() { return 8 * kvq::target_workgroups(1); }

int32_t group_shift(const kvq_cache* c) { return kvq::log2_exact(c->d.key_group); }

// Most blocks (key groups) that a workgroup of sequence i reads.
int32_t reach_of(const kvq_cache* c, int i, const Rows& r, int32_t window, int32_t sinks) {
  const int32_t seen0 = c->L[i] - r.nqry + 1, gsh = group_shift(c);
  int32_t most = 0;
  for (int first = 0; first < r.nqry; first += r.qpr) {
    const int32_t seen_first = seen0 + first, seen_last = seen0 + std::min(first + r.qpr, r.nqry) - 1;
    most = std::max(most, kvq::window_groups(seen_first, seen_last, c->Lq[i], gsh, window, sinks).count);
  }
  return most;
}

constexpr int kMinPerSplit = 4;  // 32-token blocks per split at least: one per wave

int64_t splits_bound(const kvq_cache* c) {
  const int64_t groups = c->cq / c->d.key_group;
  const int64_t per = c->split_tokens > 0 ? c->split_tokens / c->d.key_group : 1;
  return std::min<int64_t>(kvq::kMaxSplits, (groups + per - 1) / per) + 1;
}

// Estimated time of a launch, us: workgroups, 32-token blocks that a wave of the
// longest takes, bytes read, rows to merge.
double estimate_us(int64_t wgs, int64_t blocks, double bytes, int64_t merged_rows) {
  const int64_t slots = 2 * kvq::target_workgroups(1), rounds = (wgs + slots - 1) / slots;
  const double work = std::max((double)rounds * (2.0 + 0.7 * (double)blocks), bytes / 5.0e6);
  return 3.0 + work + (merged_rows > 0 ? 4.0 + 2e-3 * (double)merged_rows : 0.0);
}

struct Plan {
  Rows r;
  int32_t per = 1;                       // key groups per split
  std::vector<int32_t> nq, ns, base;     // per sequence: packed splits, all splits, first record
  int64_t records = 0;
};

Plan plan_for(const kvq_cache* c, int nqry, int32_t window, int32_t sinks) {
  Plan p;
  p.r = rows_for(c, nqry);
  const int B = c->d.batch;
  p.nq.assign(B, 0);
  p.ns.assign(B, 0);
  p.base.assign(B, 0);
  std::vector<int32_t> reach(B, 0);
  int64_t longest = 1;
  const int64_t units = units_of(c, p.r), rows = (int64_t)nqry * c->d.num_q_heads;
  double bytes = 0.0;
  for (int i = 0; i < B; ++i) {
    if (c->L[i] == 0) continue;
    reach[i] = reach_of(c, i, p.r, window, sinks);
    longest = std::max<int64_t>(longest, reach[i]);
    bytes += (double)reach[i] * c->d.key_group * 256.0 * c->d.num_kv_heads;
  }
  const int bpg = c->d.key_group / 32;
  int64_t per = longest;
  if (c->split_tokens > 0) {
    per = std::max<int64_t>(c->split_tokens / c->d.key_group, (longest + kvq::kMaxSplits - 1) / kvq::kMaxSplits);
  } else {
    double best = 0.0;
    int64_t tried = 0;
    for (int64_t ns = 1; ns <= std::min<int64_t>(kvq::kMaxSplits, longest); ++ns) {
      const int64_t n = (longest + ns - 1) / ns;
      if (n == tried) continue;
      tried = n;
      if (ns > 1 && n * bpg < kMinPerSplit) break;
      int64_t wgs = 0, merged = 0;
      for (int i = 0; i < B; ++i) {
        if (c->L[i] == 0) continue;
        const int64_t k = std::max<int64_t>(1, (reach[i] + n - 1) / n);
        wgs += units * k;
        merged += k > 1 ? rows : 0;
      }
      if (ns > 1 && wgs > most_workgroups()) break;
      const double t = estimate_us(wgs, (n * bpg + 3) / 4, bytes, merged);
      if (ns == 1 || t < best) best = t, per = n;
    }
  }
  p.per = (int32_t)per;
  int64_t wgs = 0, tails = 0;
  for (int i = 0; i < B; ++i) {
    if (c->L[i] == 0) continue;
    p.nq[i] = (int32_t)((reach[i] + per - 1) / per);
    p.ns[i] = std::max(1, p.nq[i]);
    wgs += units * p.ns[i];
    if (p.nq[i] > 1 && c->L[i] > c->Lq[i]) tails += units;
  }
  // the fp16 tail takes a workgroup of its own where there is room and the splits
  // are merged anyway
  const bool own_tails = wgs + tails <= kvq::target_workgroups(1);
  for (int i = 0; i < B; ++i) {
    if (own_tails && p.nq[i] > 1 && c->L[i] > c->Lq[i]) ++p.ns[i];
    p.base[i] = (int32_t)p.records;
    p.records += p.ns[i] > 1 ? p.ns[i] : 0;
  }
  return p;
}

size_t record_bytes(const kvq_cache* c, int nqry) {
  return (size_t)c->d.num_q_heads * nqry * kvq::kRecFloats * sizeof(float);
}

void full(const kvq_cache* c, int32_t& window, int32_t& sinks) {
  int32_t longest = 1;
  for (int i = 0; i < c->d.batch; ++i) longest = std::max(longest, c->L[i]);
  window = window < 0 ? longest : std::min(window, longest);
  sinks = std::min(sinks, longest);
}

size_t bound(const kvq_cache* c, int32_t n_q, int32_t window, int32_t sinks) {
  (void)window;
  (void)sinks;
  const int64_t each = splits_bound(c), all = c->d.batch * each;
  if (c->split_tokens > 0) return (size_t)all * record_bytes(c, n_q);
  // a plan of more than one split has most_workgroups() of them at most, and the tails'
  const int64_t most = most_workgroups() / units_of(c, rows_for(c, n_q)) + c->d.batch;
  return (size_t)std::max<int64_t>(1, std::min(all, most)) * record_bytes(c, n_q);
}

size_t need(const kvq_cache* c, int32_t n_q, int32_t window, int32_t sinks) {
  full(c, window, sinks);
  return (size_t)plan_for(c, n_q, window, sinks).records * record_bytes(c, n_q);
}

kvq_status attend(const kvq_cache* c, const void* q, int32_t n_q, int32_t window, int32_t sinks, float* out, void* ws,
                  size_t ws_bytes, void* stream) {
  const kvq_cache_desc& d = c->d;
  full(c, window, sinks);
  const Plan p = plan_for(c, n_q, window, sinks);
  const size_t bytes = (size_t)p.records * record_bytes(c, n_q);
  if (bytes > 0 && !ws) return fail(KVQ_ERR_ARG, "workspace is NULL");
  if (ws_bytes < bytes) return fail(KVQ_ERR_CAPACITY, "workspace holds %zu bytes, this call needs %zu", ws_bytes, bytes);
  if (reinterpret_cast<uintptr_t>(ws) % 16 != 0) return fail(KVQ_ERR_ARG, "workspace must be 16-byte aligned");
  int i = 0;
  while (i < d.batch) {
    kvq::DecodeArgs a{};
    const kvq::HeadLayout& lay = c->lay[0];
    a.arena = c->arena;
    a.q = static_cast<const uint16_t*>(q);
    a.ws = static_cast<float*>(ws);
    a.out = out;
    a.head_stride = lay.stride;
    a.kc = kvq::region_units(lay.kc); a.km = kvq::region_units(lay.km); a.vc = kvq::region_units(lay.vc);
    a.vm = kvq::region_units(lay.vm); a.tk = kvq::region_units(lay.tk); a.tv = kvq::region_units(lay.tv); a.vb = kvq::region_units(lay.vb);
    a.hq = d.num_q_heads; a.hkv = d.num_kv_heads; a.gk = d.key_group; a.gv = d.value_group; a.W = c->W;
    a.split_tokens = p.per * d.key_group;
    a.qscale = (float)(1.4426950408889634 / std::sqrt((double)d.head_dim));
    a.nqry = p.r.nqry; a.qpr = p.r.qpr; a.nrg = p.r.nrg; a.gqh = d.num_q_heads / d.num_kv_heads;
    a.pm = c->pm;
    a.window = window;
    a.sinks = sinks;
    int64_t wg = 0;
    for (; i < d.batch && a.nseq < kvq::kMaxSeqPerLaunch; ++i) {
      if (c->L[i] == 0) continue;
      kvq::DecodeSeq& s = a.seq[a.nseq++];
      s.head0 = c->head0[i];
      s.seq = i; s.L = s.L_old = c->L[i]; s.Lq = c->Lq[i];
      s.nq = p.nq[i]; s.nsplit = p.ns[i]; s.ws_base = p.base[i];
      s.wg_begin = (int32_t)wg;
      wg += p.ns[i] * units_of(c, p.r);
    }
    a.total_wg = (int32_t)wg;
    const int e = kvq::launch_block_tiles(a, c->type_k, c->type_v, p.r.rows, stream);
    if (e) return kvq::hip_fail(e, "block-scaled attention launch");
  }
  for (int b = 0; b < d.batch; b += kvq::kMaxSeqPerLaunch) {
    kvq::MergeArgs m{};
    m.ws = static_cast<const float*>(ws);
    m.out = out;
    m.hq = d.num_q_heads * n_q;
    for (int k = b; k < std::min(d.batch, b + kvq::kMaxSeqPerLaunch); ++k) {
      if (p.ns[k] == 1) continue;
      m.seq[m.nseq].seq = k; m.seq[m.nseq].nsplit = p.ns[k]; m.seq[m.nseq].ws_base = p.base[k];
      ++m.nseq;
    }
    const int e = kvq::launch_merge(m, stream);
    if (e) return kvq::hip_fail(e, "merge launch");
  }
  return kvq::ok();
}

// Block-scaled caches have one type pair: the classes that appends sort by are all 8 bits.
template <bool K8, bool V8>
int append(const kvq::AppendArgs& a, const kvq::RotaryArgs* rot, int, int, void* stream) {
  return kvq::launch_append_block(a, rot, K8, V8, stream);
}

template <bool K8, bool V8>
const kvq::BlockCalls* calls() {
  static const kvq::BlockCalls table = {append<K8, V8>, bound, need, attend, kvq::launch_dequant_block,
                                        kvq::launch_export_block};
  return &table;
}

// The descriptor that lengths, pages and appends go by.
struct Desc {
  kvq_cache_desc d{};
  std::vector<uint8_t> bits;
};

kvq_status convert(const kvq_block_desc* b, Desc& out) {
  if (!b) return fail(KVQ_ERR_ARG, "descriptor is NULL");
  if (b->batch < 1) return fail(KVQ_ERR_ARG, "batch must be >= 1 (got %d)", b->batch);
  for (int t : {b->type_k, b->type_v})
    if (t != KVQ_I8 && t != KVQ_E4M3) return fail(KVQ_ERR_ARG, "type %d is none of kvq_block_type", t);
  if (!(b->block_tokens == 32 || b->block_tokens == 64 || b->block_tokens == 128))
    return fail(KVQ_ERR_ARG, "block_tokens %d; must be 32, 64 or 128", b->block_tokens);
  out.bits.assign(b->batch, 8);
  kvq_cache_desc& d = out.d;
  d.batch = b->batch; d.num_q_heads = b->num_q_heads; d.num_kv_heads = b->num_kv_heads; d.head_dim = b->head_dim;
  d.max_tokens = b->max_tokens; d.key_group = b->block_tokens; d.value_group = kvq::kHeadDim;
  d.fp16_window = b->fp16_window; d.bits_k = d.bits_v = out.bits.data();
  d.page_tokens = b->page_tokens; d.num_pages = b->num_pages;
  return kvq::check_desc(&d);
}

}  // namespace

extern "C" {

size_t kvq_block_cache_bytes(const kvq_block_desc* desc) try {
  Desc d;
  return convert(desc, d) == KVQ_OK ? kvq::arena_bytes(&d.d, true) : 0;
} catch (const std::bad_alloc&) {
  kvq::no_memory();
  return 0;
}

kvq_status kvq_block_cache_init(kvq_cache** out, const kvq_block_desc* desc, void* arena, size_t arena_bytes) try {
  if (!out) return fail(KVQ_ERR_ARG, "out is NULL");
  *out = nullptr;
  Desc d;
  kvq_status st = convert(desc, d);
  if (st != KVQ_OK) return st;
  st = kvq::init_cache(out, &d.d, arena, arena_bytes, true);
  if (st != KVQ_OK) return st;
  kvq_cache* c = *out;
  c->type_k = desc->type_k;
  c->type_v = desc->type_v;
  c->block = desc->type_k == KVQ_E4M3 ? (desc->type_v == KVQ_E4M3 ? calls<true, true>() : calls<true, false>())
                                      : (desc->type_v == KVQ_E4M3 ? calls<false, true>() : calls<false, false>());
  return kvq::ok();
} catch (const std::bad_alloc&) {
  return kvq::no_memory();
}

}  // extern "C"
