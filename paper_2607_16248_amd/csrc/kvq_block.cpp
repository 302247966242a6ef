// Host side of the block-scaled caches (include/kvq.h): descriptors, the split plan
// of their attention, and its launches.  Lengths, pages and appends are the packed
// caches' (kvq_api.cpp).
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "kvq.h"
#include "kvq_host.h"
#include "kvq_internal.h"

using kvq::fail;

namespace {

// Rows of an attention launch: nqry queries per sequence in row groups of qpr
// queries (DecodeArgs): tiles of up to 16 or 32 rows, or workgroups of `waves` row
// groups of 32 (block_rows.hip).
struct Rows {
  int nqry = 1, qpr = 1, nrg = 1, rows = 16;
  int waves = 0;   // many rows: row groups per workgroup, else 0
  int groups = 1;  // that take parts of their own: row groups, or workgroups' sets of them
};

// Many rows from so many (query, head) rows of a kv head on.  32 query and 8 kv heads,
// e4m3, 16 sequences of 8000 to 16384 tokens: 64 rows 169 us in tiles and 199 in the other
// kernel, 128 rows 281 and 189; one sequence of 16384: 64 rows 40 and 43, 96 rows 42 and
// 46, 128 rows 49 and 51, 256 rows 50 and 50, 512 rows 78 and 73.  One number for both:
// between 96 and 256 rows one sequence loses up to 4 us to what a batch gains (92).
constexpr int kManyRows = 96;

Rows rows_for(const kvq_cache* c, int nqry) {
  const int gqh = c->d.num_q_heads / c->d.num_kv_heads;
  Rows r;
  r.nqry = nqry;
  r.rows = nqry * gqh > 16 ? 32 : 16;
  r.qpr = std::min(nqry, r.rows / gqh);
  r.nrg = r.groups = (nqry + r.qpr - 1) / r.qpr;
  if (nqry * gqh >= kManyRows) {
    // (five groups: 53 us with eight waves, 58 with four; three: 51 and 47)
    r.waves = r.nrg > 4 ? 8 : 4;
    r.groups = (r.nrg + r.waves - 1) / r.waves;
  }
  return r;
}

int32_t group_shift(const kvq_cache* c) { return kvq::log2_exact(c->d.key_group); }

// Units of work of the groups of a sequence: key groups (tiles, the most of any
// row group, and one for the tail) or 32-token blocks.
int32_t tile_units(const kvq_cache* c, int i, const Rows& r, int32_t window, int32_t sinks) {
  const int32_t seen0 = c->L[i] - r.nqry + 1, gsh = group_shift(c);
  int32_t most = 0;
  for (int first = 0; first < r.nqry; first += r.qpr) {
    const int32_t seen_first = seen0 + first, seen_last = seen0 + std::min(first + r.qpr, r.nqry) - 1;
    most = std::max(most, kvq::window_groups(seen_first, seen_last, c->Lq[i], gsh, window, sinks).count);
  }
  return most + (c->L[i] > c->Lq[i] ? 1 : 0);
}
int32_t row_units(const kvq_cache* c, int i, const Rows& r, int32_t window, int32_t sinks, int group) {
  return kvq::row_blocks(r.nqry, r.qpr * r.waves, c->L[i], c->Lq[i], group_shift(c), window, sinks, group).total;
}

// Workgroups of a launch, where there is work for so many: as many as are resident.
int64_t workgroups(const Rows& r) { return (r.waves == 8 ? 1 : 2) * kvq::target_workgroups(1); }
constexpr int64_t kMostWorkgroups = ((int64_t)1 << 22) - 1;  // of up to 512 threads: a launch's threads stay below 2^32
constexpr int kMinBlocks = 4;  // 32-token blocks per workgroup at least (tiles: one per wave)

// Tiles: units that stand for a row group's beginning and end (queries, joined waves,
// records) and its fp16 tail, in the time of a key group each: kPartTokens tokens, the
// tail's and 64 more.  64 sequences of 100 to 12000 tokens, tails of 128 to 191: 184 us
// without them, 150 with 256 tokens, 140 with 384 and with 768.  Where a workgroup's
// share is small, every one has a beginning and an end, and they count for a quarter
// of it at most.
constexpr int kPartTokens = 384;
int32_t tile_extra(int32_t tail, int32_t G, int64_t share) {
  const int64_t tokens = std::min<int64_t>((tail > 0 ? tail + 64 - G : 0) + kPartTokens, share * G / 4);
  return std::max(0, (int32_t)((tokens + G - 1) / G));
}
// Many rows: the same, in blocks.  512 rows of 5 sequences of 300 to 16384 tokens, 384 of
// 16 of 2000 to 16384: 302 us without them, 173 and 482 with 8, 143 and 491 with 16, 144
// and 515 with 32.
constexpr int kRowExtra = 16;

// What a call's launches are given: the list of work units of a launch's sequences, of
// which every workgroup takes `per`.
struct Plan {
  Rows r;
  std::vector<int32_t> real, units, begin, ns, base;  // per sequence: DecodeSeq's L_old, nq, wg_begin, nsplit, ws_base
  std::vector<int> first;                             // per launch: its first sequence
  std::vector<int32_t> per, total, extra;             // per launch
  int64_t records = 0;
  bool fits = true;
};

Plan plan_for(const kvq_cache* c, int nqry, int32_t window, int32_t sinks) {
  Plan p;
  p.r = rows_for(c, nqry);
  const Rows& r = p.r;
  const int B = c->d.batch, G = c->d.key_group, hkv = c->d.num_kv_heads;
  for (auto* v : {&p.real, &p.units, &p.begin, &p.ns, &p.base}) v->assign(B, 0);
  for (int i = 0; i < B;) {
    const int from = i;
    p.first.push_back(i);
    int64_t total = 0;
    for (int n = 0; i < B && n < kvq::kMaxSeqPerLaunch; ++i) {
      if (c->L[i] == 0) continue;
      ++n;
      if (r.waves) {
        for (int g = 0; g < r.groups; ++g) p.real[i] += row_units(c, i, r, window, sinks, g);
        total += (int64_t)hkv * p.real[i];
      } else {
        p.real[i] = tile_units(c, i, r, window, sinks);
        total += (int64_t)hkv * r.groups * p.real[i];
      }
    }
    const int64_t share = (total + workgroups(r) - 1) / workgroups(r);
    const int32_t extra = (int32_t)std::min<int64_t>(kRowExtra, share / 4);
    total = 0;
    for (int k = from; k < i; ++k) {
      if (c->L[k] == 0) continue;
      p.units[k] = p.real[k] + (r.waves ? r.groups * extra : tile_extra(c->L[k] - c->Lq[k], G, share));
      p.begin[k] = (int32_t)std::min<int64_t>(total, INT32_MAX);
      total += (int64_t)hkv * (r.waves ? 1 : r.groups) * p.units[k];
    }
    const int64_t least = r.waves ? kMinBlocks : (kMinBlocks * 32 + G - 1) / G;
    int64_t per = std::max<int64_t>({(total + workgroups(r) - 1) / workgroups(r), least, 1});
    // (forced splits: as many as one launch takes at most, longer ones where there would be more)
    if (c->split_tokens > 0) per = std::max<int64_t>(c->split_tokens / (r.waves ? 32 : G), (total + kMostWorkgroups - 1) / kMostWorkgroups);
    p.fits &= total + per < INT32_MAX;
    p.per.push_back((int32_t)per);
    p.extra.push_back(extra);
    p.total.push_back((int32_t)std::min<int64_t>(total, INT32_MAX));
    for (int k = from; k < i && p.fits; ++k) {
      if (c->L[k] == 0) continue;
      // parts of the group with the most of them
      int64_t ns = 1, b = p.begin[k];
      for (int h = 0; h < hkv; ++h)
        for (int g = 0; g < r.groups; ++g) {
          const int64_t n = r.waves ? row_units(c, k, r, window, sinks, g) : p.real[k];
          ns = std::max(ns, (b + n - 1) / per - b / per + 1);
          b += r.waves ? n + extra : p.units[k];
        }
      p.ns[k] = (int32_t)ns;
      p.base[k] = (int32_t)std::min<int64_t>(p.records, INT32_MAX);
      p.records += ns > 1 ? ns : 0;
    }
  }
  p.fits &= p.records < INT32_MAX;
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

// A group of n units in parts of `per` has (n + per - 2) / per + 1 of them at most.
size_t bound(const kvq_cache* c, int32_t n_q, int32_t window, int32_t sinks) {
  (void)window;
  (void)sinks;
  const Rows r = rows_for(c, n_q);
  const int64_t G = c->d.key_group, B = c->d.batch, unit = r.waves ? 32 : G;
  const int64_t units = ((int64_t)c->d.max_tokens + unit - 1) / unit + 2;  // of a group, without those that stand for no work
  const int64_t least = c->split_tokens > 0 ? c->split_tokens / unit
                                            : std::max<int64_t>(1, r.waves ? kMinBlocks : (kMinBlocks * 32 + G - 1) / G);
  int64_t records = B * ((units + least - 2) / least + 1);
  if (c->split_tokens == 0) {
    // per >= total / workgroups: of the sequences of a launch, the sum of units / per over all
    // groups is workgroups() at most, and a group has no more parts than that and 2.
    // Many rows: the group with the most blocks counts; half of them are the average at least
    // (causal groups grow evenly), and the kv heads have them all
    const int64_t launches = (B + kvq::kMaxSeqPerLaunch - 1) / kvq::kMaxSeqPerLaunch;
    const int64_t groups = (int64_t)c->d.num_kv_heads * r.groups;
    records = std::min(records, launches * ((r.waves ? 2 : 1) * workgroups(r) / groups + 1) + 3 * B);
  }
  return (size_t)std::max<int64_t>(1, records) * record_bytes(c, n_q);
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
  if (!p.fits) return fail(KVQ_ERR_UNSUPPORTED, "too much work for one call");
  const size_t bytes = (size_t)p.records * record_bytes(c, n_q);
  if (bytes > 0 && !ws) return fail(KVQ_ERR_ARG, "workspace is NULL");
  if (ws_bytes < bytes) return fail(KVQ_ERR_CAPACITY, "workspace holds %zu bytes, this call needs %zu", ws_bytes, bytes);
  if (reinterpret_cast<uintptr_t>(ws) % 16 != 0) return fail(KVQ_ERR_ARG, "workspace must be 16-byte aligned");
  for (size_t k = 0; k < p.first.size(); ++k) {
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
    a.units_per_wg = p.per[k];
    a.extra_units = p.extra[k];
    a.qscale = (float)(1.4426950408889634 / std::sqrt((double)d.head_dim));
    a.nqry = p.r.nqry; a.qpr = p.r.qpr; a.nrg = p.r.nrg; a.gqh = d.num_q_heads / d.num_kv_heads;
    a.pm = c->pm;
    a.window = window;
    a.sinks = sinks;
    for (int i = p.first[k]; i < d.batch && a.nseq < kvq::kMaxSeqPerLaunch; ++i) {
      if (c->L[i] == 0) continue;
      kvq::DecodeSeq& s = a.seq[a.nseq++];
      s.head0 = c->head0[i];
      s.seq = i; s.L = c->L[i]; s.Lq = c->Lq[i];
      s.L_old = p.real[i];
      s.nq = p.units[i]; s.nsplit = p.ns[i]; s.ws_base = p.base[i];
      s.wg_begin = p.begin[i];
    }
    a.total_wg = p.total[k];  // units
    const int e = p.r.waves ? kvq::launch_block_rows(a, c->type_k, c->type_v, p.r.waves, stream)
                            : kvq::launch_block_tiles(a, c->type_k, c->type_v, p.r.rows, stream);
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
