// C ABI of the packed low-bit KV-cache library: argument checks, host-side
// length bookkeeping, the split plan of the decode kernel, and launches.
//
// Everything before a launch is plain host code that touches no device and
// calls no HIP function, so argument and capacity errors are detected (and
// testable) without a GPU and leave the cache unchanged.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <map>
#include <memory>
#include <new>
#include <string>
#include <utility>
#include <vector>

#include "dgap.h"
#include "kvq.h"
#include "kvq_host.h"
#include "kvq_internal.h"
#include "kvq_layout.h"

using kvq::HeadLayout;
using kvq::check_rows;
using kvq::fail;
using kvq::hip_fail;
using kvq::kMaxSplits;
using kvq::log2_exact;
using kvq::no_memory;
using kvq::ok;
using kvq::packed_len;
using kvq::target_workgroups;

static_assert(kvq::kScratchBytes == KVQ_NOALLOC_SCRATCH_BYTES, "scratch array size as the header states");
static_assert(kvq::kDistillMaxK == DGAP_MAX_TEACHER, "teacher entries as the header states");
static_assert(kvq::kSpareRow >= KVQ_MAX_CHUNK, "a spare row lies past every chunk query");

namespace kvq {

namespace {
thread_local std::string g_err;
}  // namespace

// Decode workgroups that fit the current device at once (one round of the
// grid): compute units times the resident workgroups per unit (one 4-wave
// workgroup per wave slot of a SIMD).
int64_t target_workgroups(int per_cu) {
  static thread_local int cached_dev = -1;
  static thread_local int64_t cus = 0;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 256 * per_cu;
  if (dev != cached_dev) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    cached_dev = dev;
    cus = n;
  }
  return cus * per_cu;
}

kvq_status fail(kvq_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  try {
    g_err = buf;
  } catch (const std::bad_alloc&) {
    g_err.clear();
  }
  return s;
}
// What a call of the C interface ends with when its plan finds no memory: no exception
// may pass it.
kvq_status no_memory() { return fail(KVQ_ERR_CAPACITY, "no host memory"); }

kvq_status ok() {
  g_err.clear();
  return KVQ_OK;
}
const char* last_error() { return g_err.c_str(); }

int64_t packed_capacity(const kvq_cache_desc* d) {
  const int64_t past = (int64_t)d->max_tokens - d->fp16_window;
  return past <= 0 ? 0 : past / d->key_group * d->key_group;
}

int32_t quantized_len(int64_t L, const kvq_cache_desc& d) {
  const int64_t past = L - d.fp16_window;
  return past <= 0 ? 0 : (int32_t)(past / d.key_group * d.key_group);
}

int log2_exact(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}

kvq_status hip_fail(int e, const char* what) {
  return fail(KVQ_ERR_HIP, "%s: %s", what, hipGetErrorString((hipError_t)e));
}

static bool valid_bits(int b) { return b == 1 || b == 2 || b == 4 || b == 8; }

kvq_status check_desc(const kvq_cache_desc* d) {
  if (!d) return fail(KVQ_ERR_ARG, "descriptor is NULL");
  if (d->batch < 1) return fail(KVQ_ERR_ARG, "batch must be >= 1 (got %d)", d->batch);
  if (d->num_kv_heads < 1) return fail(KVQ_ERR_ARG, "num_kv_heads must be >= 1");
  if (d->num_q_heads < 1 || d->num_q_heads % d->num_kv_heads != 0)
    return fail(KVQ_ERR_ARG, "num_q_heads (%d) must be a positive multiple of num_kv_heads (%d)",
                d->num_q_heads, d->num_kv_heads);
  const int gq = d->num_q_heads / d->num_kv_heads;
  if (!(gq == 1 || gq == 2 || gq == 4 || gq == 5 || gq == 8))
    return fail(KVQ_ERR_UNSUPPORTED, "num_q_heads / num_kv_heads = %d; supported: 1, 2, 4, 5, 8", gq);
  if (d->head_dim < 1) return fail(KVQ_ERR_ARG, "head_dim must be positive");
  if (d->head_dim != kvq::kHeadDim) return fail(KVQ_ERR_UNSUPPORTED, "head_dim %d; only 128 is supported", d->head_dim);
  if (d->max_tokens < 1) return fail(KVQ_ERR_ARG, "max_tokens must be >= 1");
  if (!(d->key_group == 32 || d->key_group == 64 || d->key_group == 128))
    return fail(KVQ_ERR_ARG, "key_group %d; must be 32, 64 or 128", d->key_group);
  const int gv = d->value_group;
  if (!(gv == 8 || gv == 16 || gv == 32 || gv == 64 || gv == 128))
    return fail(KVQ_ERR_ARG, "value_group %d; must be 8, 16, 32, 64 or 128", gv);
  if (d->fp16_window < 0) return fail(KVQ_ERR_ARG, "fp16_window must be >= 0");
  if ((int64_t)d->fp16_window + d->key_group > (int64_t)1 << 30) return fail(KVQ_ERR_ARG, "fp16_window too large");
  if (!d->bits_k || !d->bits_v) return fail(KVQ_ERR_ARG, "bits_k and bits_v must be host arrays of length batch");
  for (int i = 0; i < d->batch; ++i) {
    if (!valid_bits(d->bits_k[i]) || !valid_bits(d->bits_v[i]))
      return fail(KVQ_ERR_ARG, "sequence %d: bits (%d, %d) must each be 1, 2, 4 or 8", i, d->bits_k[i], d->bits_v[i]);
  }
  const int P = d->page_tokens;
  if (P < 0 || (P > 0 && (P < d->key_group || P > (1 << 20) || (P & (P - 1)) != 0)))
    return fail(KVQ_ERR_ARG, "page_tokens %d: must be 0 or a power of two in [key_group = %d, 2^20]", P, d->key_group);
  if (d->num_pages < 0 || (d->num_pages > 0 && P == 0))
    return fail(KVQ_ERR_ARG, "num_pages %d: must be >= 0, and 0 unless page_tokens > 0", d->num_pages);
  if (P > 0) {
    for (int i = 1; i < d->batch; ++i)
      if (d->bits_k[i] != d->bits_k[0] || d->bits_v[i] != d->bits_v[0])
        return fail(KVQ_ERR_UNSUPPORTED, "a paged cache needs one bit width pair for every sequence");
  }
  return KVQ_OK;
}

// Rows of logits that a call reads whole.
kvq_status check_rows(const void* logits, int type, int64_t row_stride, int rows, int vocab, const char* what) {
  if (!logits) return fail(KVQ_ERR_ARG, "logits is NULL");
  if (type != DGAP_F32 && type != DGAP_F16 && type != DGAP_BF16) return fail(KVQ_ERR_ARG, "type %d is none of dgap_type", type);
  if (rows < 1) return fail(KVQ_ERR_ARG, "%s must be >= 1 (got %d)", what, rows);
  if (vocab < 1) return fail(KVQ_ERR_ARG, "vocab must be >= 1 (got %d)", vocab);
  if (vocab > 1 << 24) return fail(KVQ_ERR_UNSUPPORTED, "vocab %d above 2^24", vocab);
  if (row_stride < vocab) return fail(KVQ_ERR_ARG, "row_stride %lld smaller than vocab %d", (long long)row_stride, vocab);
  // (a launch's threads, up to 1024 for 8192 logits, stay below 2^32)
  if ((int64_t)rows * ((vocab + 8191) / 8192) >= (int64_t)1 << 22)
    return fail(KVQ_ERR_UNSUPPORTED, "%d rows of %d logits are too many for one call", rows, vocab);
  const int size = type == DGAP_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(logits) % size != 0) return fail(KVQ_ERR_ARG, "logits must be aligned to their type");
  return KVQ_OK;
}

}  // namespace kvq

namespace {

using kvq::check_desc;
using kvq::packed_capacity;
using kvq::quantized_len;

constexpr int kMinGroupsPerSplit = 4;    // one key group per wave at least
// Layout of `tokens` packed tokens and `w` ring slots of a head.
HeadLayout layout_for(const kvq_cache_desc* d, int bk, int bv, int64_t tokens, int64_t w, bool with_bound, bool block) {
  return block ? kvq::block_layout(tokens, d->key_group, w, with_bound)
               : kvq::head_layout(bk, bv, tokens, d->key_group, d->value_group, w, with_bound);
}
HeadLayout layout_of(const kvq_cache_desc* d, int bk, int bv, bool block) {
  return layout_for(d, bk, bv, packed_capacity(d), (int64_t)d->fp16_window + d->key_group, true, block);
}

// Arena of a paged cache: header | fp16 rings [batch][Hkv] | block table
// [batch][max_pages] int32 | pool [num_pages][Hkv][page head layout].
struct PagedArena {
  HeadLayout page, ring, seq_lay;  // seq_lay: packed offsets of the page, ring offsets and stride
  uint64_t table_off = 0, pool0 = 0, page_bytes = 0, total = 0;
  int32_t max_pages = 0, num_pages = 0;
};

PagedArena paged_arena(const kvq_cache_desc* d, bool block) {
  PagedArena A;
  const int bk = d->bits_k[0], bv = d->bits_v[0], P = d->page_tokens;
  const int64_t W = (int64_t)d->fp16_window + d->key_group;
  A.page = layout_for(d, bk, bv, P, 0, false, block);
  A.ring = layout_for(d, bk, bv, 0, W, true, block);
  A.seq_lay = A.page;
  A.seq_lay.tk = A.ring.tk;
  A.seq_lay.tv = A.ring.tv;
  A.seq_lay.vb = A.ring.vb;
  A.seq_lay.stride = A.ring.stride;
  A.max_pages = (int32_t)((packed_capacity(d) + P - 1) / P);
  A.num_pages = d->num_pages > 0 ? d->num_pages : d->batch * A.max_pages;
  const uint64_t rings = (uint64_t)d->batch * d->num_kv_heads * A.ring.stride;
  A.table_off = kvq::align_up(kvq::kHeaderBytes + rings, kvq::kAlign);
  A.pool0 = kvq::align_up(A.table_off + (uint64_t)d->batch * A.max_pages * 4, kvq::kAlign);
  A.page_bytes = (uint64_t)d->num_kv_heads * A.page.stride;
  A.total = A.pool0 + (uint64_t)A.num_pages * A.page_bytes;
  return A;
}

// Split length of one launch's sequences (one bit class): the launch fills
// two workgroups per compute unit (two waves per SIMD), a full round of
// the kernels that fit two and part of one for those that fit three or
// four.  Longer splits with fewer waves measured as fast or faster there:
// every wave pays a prologue (query, zero-point table, first loads) and an
// epilogue, all waves' first loads queue behind each other, and the merge
// reads fewer records.  Fewer than two per unit (one wave per SIMD on some
// units) measured 15-36% slower.  Classes launch one after another, so each
// gets the whole device.
int32_t split_tokens_for(const kvq_cache* c, const std::vector<int>& seqs, int nqry, int nrg, int occ_rows) {
  const int gk = c->d.key_group;
  if (c->split_tokens > 0) return c->split_tokens;
  int64_t total = 0, lq_max = 0, tails = 0;
  int occ = 4;
  for (int i : seqs) {
    total += (int64_t)c->Lq[i] * c->d.num_kv_heads * nrg;
    lq_max = std::max<int64_t>(lq_max, c->Lq[i]);
    if (c->L[i] > c->Lq[i]) tails += (int64_t)c->d.num_kv_heads * nrg;
    occ = std::min(occ, occ_rows > 0 && c->matrix[i] ? occ_rows : c->occupancy[i]);
  }
  // The fp16-tail workgroups (one per sequence and kv head with tail tokens)
  // must not wait for a free slot (that would add a whole split's time to
  // the launch).  Single-token decode of one sequence with kernels that fit
  // more than two workgroups per compute unit takes a full round of packed
  // splits (whole blocks per wave) and its tail workgroups, a few tokens
  // each and last in id order, in spare slots; otherwise the round leaves
  // them room (with several sequences each one's tail workgroups follow its
  // own packed splits, so the ids past the round would be packed splits;
  // chunk queries' tail workgroups hold the queries' own tokens: started
  // last, they would end last).
  const int64_t round = target_workgroups(std::min(occ, 2));
  const bool tails_spare = nqry == 1 && occ > 2 && seqs.size() == 1;
  const int64_t target = tails_spare ? round : std::max<int64_t>(round - tails, round / 2);
  int64_t st = (total + target - 1) / target;
  if (nrg > 1 && !seqs.empty()) {
    // chunk queries: every row group of a (kv head, split) unit reads the
    // unit's tokens; units of at most ~1 MiB let the row groups that share
    // an XCD find them in its L2 (more workgroup rounds instead)
    const int i0 = seqs[0];
    const int64_t tok_bytes = 16 * (c->bk[i0] + c->bv[i0]) + 512 / gk + 4 * (kvq::kHeadDim / c->d.value_group);
    st = std::min<int64_t>(st, ((int64_t)1 << 20) / tok_bytes);
  }
  st = std::max<int64_t>(st, (lq_max + kMaxSplits - 1) / kMaxSplits);
  st = (st + gk - 1) / gk * gk;
  st = std::max<int64_t>(st, (int64_t)gk * kMinGroupsPerSplit);
  if (nrg == 1) {
    // Short sequences: two 32-token blocks per wave at least, while the
    // launch still gives every compute unit a workgroup (a wave's first
    // loads and its epilogue cost about as much as a block)
    const int64_t two = ((int64_t)2 * 32 * kMinGroupsPerSplit + gk - 1) / gk * gk;
    if (two > st && (total + two - 1) / two >= round / 2) st = two;
  }
  return (int32_t)std::min<int64_t>(st, (int64_t)1 << 30);
}

int64_t splits_bound(const kvq_cache* c) {
  const int64_t cq = c->cq;
  int64_t nq;
  if (c->split_tokens > 0)
    nq = (cq + c->split_tokens - 1) / c->split_tokens;
  else
    nq = std::min<int64_t>(kMaxSplits, (cq + (int64_t)c->d.key_group * kMinGroupsPerSplit - 1) /
                                           ((int64_t)c->d.key_group * kMinGroupsPerSplit));
  return nq + 1;
}

// Sequences grouped by (key bits, value bits), each class in chunks that fit
// one kernel-argument block.
std::vector<std::pair<std::pair<int, int>, std::vector<int>>> bit_classes(const kvq_cache* c,
                                                                          const std::vector<int>& seqs) {
  std::map<std::pair<int, int>, std::vector<int>> m;
  for (int i : seqs) m[{c->bk[i], c->bv[i]}].push_back(i);
  std::vector<std::pair<std::pair<int, int>, std::vector<int>>> out;
  for (auto& kv : m) {
    for (size_t b = 0; b < kv.second.size(); b += kvq::kMaxSeqPerLaunch) {
      const size_t e = std::min(kv.second.size(), b + kvq::kMaxSeqPerLaunch);
      out.push_back({kv.first, std::vector<int>(kv.second.begin() + b, kv.second.begin() + e)});
    }
  }
  return out;
}

kvq_status check_scratch(const void* ws, size_t ws_bytes, size_t need) {
  if (!ws) return fail(KVQ_ERR_ARG, "workspace is NULL");
  if (ws_bytes < need) return fail(KVQ_ERR_CAPACITY, "workspace holds %zu bytes, this call needs %zu", ws_bytes, need);
  if (reinterpret_cast<uintptr_t>(ws) % 16 != 0) return fail(KVQ_ERR_ARG, "workspace must be 16-byte aligned");
  return KVQ_OK;
}

// A workgroup per row takes all steps of a draw from so many rows on, and for
// vocabularies up to kSampleSmall: 128 rows of 128256 fp32 59 us, with chunks of
// rows 66 (64 rows 45 and 38).  Below kSampleRows, fp32: rows of 16384, 1 of them 17.8
// us and 19.9, 64 41 and 43; of 32768, 1 17.5 and 17.0, 16 20.4 and 21.0, 64 flat ones
// 27 and 31; of 40960, 1 23.5 and 20.7, 16 24.2 and 22.9, 64 25.6 and 27.4; of 50257,
// 1 21.0 and 16.6, 64 40.6 and 40.2; of 65536, 1 28 and 22, 64 43 and 41 (bf16 within
// 10% of these).
constexpr int kSampleRows = 128, kSampleSmall = 32768;

// Workspace of one row of dgap_sample (see SampleArgs::ws).
uint64_t sample_row_bytes(int vocab) {
  const uint64_t nchunk = (vocab + kvq::kSampleChunk - 1) / kvq::kSampleChunk;
  const uint64_t ngroup = (vocab + kvq::kSampleGroup - 1) / kvq::kSampleGroup;
  return kvq::align_up(12 * kvq::kSampleBins + 4 * (ngroup + nchunk), kvq::kAlign);
}

// Whether loss and gradient of rows that fit a workgroup's registers come from one
// pass over them, else from three launches that read them twice.  One pass for
// short rows, whose three launches cost more than their work (16384: 64 fp32 11 us
// and 16, bf16 512 20 and 18; 32768: 64 fp32 13 and 16, 256 19 and 24, 1024 57 and 68,
// bf16 64 12 and 15, 256 14 and 17, 512 28 and 25; 40960: 64 fp32 17.5 and 16, 256 24
// and 28, bf16 64 16 and 15.5, 256 19 and 19; 50257: 64 fp32 18 and 16, 256 26 and 32,
// bf16 64 20 and 16, 256 23 and 22; 65536: 64 fp32 20 and 17, 256 30 and 38, bf16 64
// 18 and 16, 512 35 and 40), and for
// more logits than stay in the 256 MiB cache beside their gradient (128256 bf16: 3000
// rows 335 us and 438, 1024 127 and 157, 512, which are 131 MB, 68 and 69, 128 23 and
// 24 but 64 30 and 19; 152064 f16 with 256 entries: 512, 156 MB, 98 and 83, 1024 175
// and 197).  The loss alone reads them once either way, faster by chunks (3000 rows
// of 128256 bf16 137 us and 191).
bool distill_whole_rows(int type, int64_t rows, int64_t vocab) {
  const bool f32 = type == DGAP_F32;
  if (vocab < 8 || vocab > (f32 ? kvq::kDistillRow32 : kvq::kDistillRow16)) return false;
  return vocab <= 32768 || rows * vocab * (f32 ? 4 : 2) > (int64_t)192 << 20;
}

kvq_status distill_args(kvq::DistillArgs& a, const dgap_distillation* p, void* grad, int64_t grad_row_stride,
                        const float* grad_loss, bool need_grad) {
  if (!p) return fail(KVQ_ERR_ARG, "parameters are NULL");
  const kvq_status st = check_rows(p->logits, p->type, p->row_stride, p->rows, p->vocab, "rows");
  if (st != KVQ_OK) return st;
  if (!p->teacher || !p->index) return fail(KVQ_ERR_ARG, "teacher and index must be device pointers");
  if (p->k < 1 || p->k > DGAP_MAX_TEACHER) return fail(KVQ_ERR_ARG, "k = %d outside [1, %d]", p->k, DGAP_MAX_TEACHER);
  if (!(p->temperature > 0.f) || !std::isfinite(p->temperature) || !std::isfinite(1.4426950408889634f / p->temperature))
    return fail(KVQ_ERR_ARG, "temperature %g must be positive and finite, its reciprocal too", (double)p->temperature);
  if (!grad && need_grad) return fail(KVQ_ERR_ARG, "grad must be a device pointer");
  if (grad && grad_row_stride < p->vocab)
    return fail(KVQ_ERR_ARG, "grad_row_stride %lld smaller than vocab %d", (long long)grad_row_stride, p->vocab);
  if (reinterpret_cast<uintptr_t>(grad) % (p->type == DGAP_F32 ? 4 : 2) != 0)
    return fail(KVQ_ERR_ARG, "grad must be aligned to its type");
  if (grad == p->logits && grad && grad_row_stride != p->row_stride)
    return fail(KVQ_ERR_ARG, "a gradient in the logits' place needs their row stride");
  a.logits = p->logits;
  a.teacher = p->teacher;
  a.index = p->index;
  a.grad_loss = grad_loss;
  a.grad = grad;
  a.row_stride = p->row_stride;
  a.grad_stride = grad_row_stride;
  a.rows = p->rows; a.vocab = p->vocab; a.k = p->k;
  a.nchunk = (p->vocab + kvq::kDistillChunk - 1) / kvq::kDistillChunk;
  a.whole_rows = grad && !need_grad && distill_whole_rows(p->type, p->rows, p->vocab);
  a.compute_units = (int32_t)target_workgroups(1);
  a.temperature = p->temperature;
  a.c = (float)(1.4426950408889634 / (double)p->temperature);
  return KVQ_OK;
}

}  // namespace

namespace kvq {
int matrix_decode_occupancy(int bk, int bv, int gk, int gq) { return matrix_waves(bk, bv, gk / 32, gq); }

bool window_rows_supported(int gq, int gk, int gv, uint64_t head_bytes) {
  return matrix_heads(gq, gk) && gv >= 32 && head_bytes <= 0xFFFFFFFFull;
}
bool matrix_decode_supported(int bk, int bv, int gq, int gk, int gv, uint64_t head_bytes) {
  return matrix_bits(bk, bv) && window_rows_supported(gq, gk, gv, head_bytes);
}
}  // namespace kvq

namespace kvq {

size_t arena_bytes(const kvq_cache_desc* d, bool block) {
  if (check_desc(d) != KVQ_OK) return 0;
  if (d->page_tokens > 0) return (size_t)paged_arena(d, block).total;
  uint64_t total = kvq::kHeaderBytes;
  for (int i = 0; i < d->batch; ++i) total += (uint64_t)d->num_kv_heads * layout_of(d, d->bits_k[i], d->bits_v[i], block).stride;
  return (size_t)total;
}

kvq_status init_cache(kvq_cache** out, const kvq_cache_desc* d, void* arena, size_t bytes, bool block) {
  if (!out) return fail(KVQ_ERR_ARG, "out is NULL");
  *out = nullptr;
  const kvq_status st = check_desc(d);
  if (st != KVQ_OK) return st;
  if (!arena) return fail(KVQ_ERR_ARG, "arena is NULL");
  if (reinterpret_cast<uintptr_t>(arena) % kvq::kAlign != 0) return fail(KVQ_ERR_ARG, "arena must be 256-byte aligned");
  const size_t need = arena_bytes(d, block);
  if (bytes < need)
    return fail(KVQ_ERR_CAPACITY, "arena holds %zu bytes, the cache needs %zu", bytes, need);
  std::unique_ptr<kvq_cache> owner(new kvq_cache());
  kvq_cache* c = owner.get();
  c->d = *d;
  c->bk.assign(d->bits_k, d->bits_k + d->batch);
  c->bv.assign(d->bits_v, d->bits_v + d->batch);
  c->d.bits_k = c->bk.data();
  c->d.bits_v = c->bv.data();
  c->arena = static_cast<uint8_t*>(arena);
  c->arena_bytes = bytes;
  c->cq = packed_capacity(d);
  c->W = d->fp16_window + d->key_group;
  uint64_t off = kvq::kHeaderBytes;
  uint64_t packed_bytes = 0;  // what the matrix kernel's 32-bit offsets must reach (one buffer resource)
  if (d->page_tokens > 0) {
    const PagedArena A = paged_arena(d, block);
    c->paged = true;
    c->pm.table = reinterpret_cast<const int32_t*>(c->arena + A.table_off);
    c->pm.pool0 = A.pool0;
    c->pm.page_bytes = A.page_bytes;
    c->pm.page_head_bytes = A.page.stride;
    c->pm.pool_bytes = (uint64_t)A.num_pages * A.page_bytes;
    c->pm.page_tokens = d->page_tokens;
    c->pm.max_pages = A.max_pages;
    c->pm.page_shift = log2_exact(d->page_tokens);
    c->pm.gk_shift = log2_exact(d->key_group);
    for (int i = 0; i < d->batch; ++i) {
      c->lay.push_back(A.seq_lay);
      c->head0.push_back(off);
      off += (uint64_t)d->num_kv_heads * A.ring.stride;
    }
    c->pages.assign(d->batch, {});
    for (int pg = A.num_pages - 1; pg >= 0; --pg) c->free_pages.push_back(pg);
    packed_bytes = A.page.stride;  // one page's region of one kv head, whatever the pool size
  } else {
    for (int i = 0; i < d->batch; ++i) {
      c->lay.push_back(layout_of(d, c->bk[i], c->bv[i], block));
      c->head0.push_back(off);
      off += (uint64_t)d->num_kv_heads * c->lay.back().stride;
    }
  }
  c->L.assign(d->batch, 0);
  c->Lq.assign(d->batch, 0);
  for (int i = 0; i < d->batch; ++i) {
    const int gq = d->num_q_heads / d->num_kv_heads;
    const uint64_t head_bytes = c->paged ? packed_bytes : c->lay[i].stride;
    c->matrix.push_back(kvq::matrix_decode_supported(c->bk[i], c->bv[i], gq, d->key_group, d->value_group, head_bytes) ? 1 : 0);
    c->window.push_back(kvq::window_rows_supported(gq, d->key_group, d->value_group, head_bytes) ? 1 : 0);
    auto same = [&](const std::pair<int, int>& cl) { return c->bk[cl.first] == c->bk[i] && c->bv[cl.first] == c->bv[i]; };
    const auto cl = std::find_if(c->classes.begin(), c->classes.end(), same);
    if (cl == c->classes.end()) c->classes.push_back({i, 1});
    else ++cl->second;
  }
  // the split plan of a launch fills one round of its kernel's workgroups
  for (int i = 0; i < d->batch; ++i)
    c->occupancy.push_back(c->matrix[i] ? kvq::matrix_decode_occupancy(c->bk[i], c->bv[i], d->key_group,
                                                                       d->num_q_heads / d->num_kv_heads)
                                        : 2);
  *out = owner.release();
  return ok();
}

}  // namespace kvq

extern "C" {

size_t kvq_cache_bytes(const kvq_cache_desc* d) { return kvq::arena_bytes(d, false); }

kvq_status kvq_cache_init(kvq_cache** out, const kvq_cache_desc* d, void* arena, size_t arena_bytes) try {
  return kvq::init_cache(out, d, arena, arena_bytes, false);
} catch (const std::bad_alloc&) {
  return no_memory();
}

void kvq_cache_destroy(kvq_cache* c) { delete c; }

kvq_status kvq_cache_reset(kvq_cache* c, void* stream) {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  const int e = kvq::launch_fill_zero(c->arena, kvq::kHeaderBytes / 4, stream);
  if (e) return hip_fail(e, "reset");
  std::fill(c->L.begin(), c->L.end(), 0);
  std::fill(c->Lq.begin(), c->Lq.end(), 0);
  if (c->paged) {
    for (auto& pl : c->pages) {
      for (int32_t pg : pl) c->free_pages.push_back(pg);
      pl.clear();
    }
  }
  return ok();
}

int64_t kvq_seq_len(const kvq_cache* c, int32_t seq) {
  if (!c || seq < 0 || seq >= c->d.batch) return -1;
  return c->L[seq];
}

kvq_status kvq_seq_release(kvq_cache* c, int32_t seq) {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (seq < 0 || seq >= c->d.batch) return fail(KVQ_ERR_ARG, "seq %d out of range", seq);
  c->L[seq] = 0;
  c->Lq[seq] = 0;
  if (c->paged) {
    for (int32_t pg : c->pages[seq]) c->free_pages.push_back(pg);
    c->pages[seq].clear();
  }
  return ok();
}

int64_t kvq_free_pages(const kvq_cache* c) {
  if (!c || !c->paged) return -1;
  return (int64_t)c->free_pages.size();
}

kvq_status kvq_truncate(kvq_cache* c, const int32_t* lens) {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (!lens) return fail(KVQ_ERR_ARG, "lens is NULL");
  for (int i = 0; i < c->d.batch; ++i) {
    if (lens[i] < 0 || lens[i] > c->L[i])
      return fail(KVQ_ERR_ARG, "sequence %d: length %d outside [0, %d]", i, lens[i], c->L[i]);
    if (lens[i] < c->Lq[i])
      return fail(KVQ_ERR_STATE, "sequence %d: length %d is below its %d packed tokens", i, lens[i], c->Lq[i]);
  }
  std::copy(lens, lens + c->d.batch, c->L.begin());
  return ok();
}

}  // extern "C"

namespace kvq {

kvq_status append_tokens(kvq_cache* c, const void* K, const void* V, int32_t n_max, const int32_t* n_new,
                         const RotaryArgs* rot, AppendLaunch launch, void* stream) {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (!n_new) return fail(KVQ_ERR_ARG, "n_new is NULL");
  if (n_max < 0) return fail(KVQ_ERR_ARG, "n_max must be >= 0");
  const kvq_cache_desc& d = c->d;
  bool any = false;
  for (int i = 0; i < d.batch; ++i) {
    if (n_new[i] < 0 || n_new[i] > n_max)
      return fail(KVQ_ERR_ARG, "sequence %d: n_new = %d outside [0, n_max = %d]", i, n_new[i], n_max);
    if ((int64_t)c->L[i] + n_new[i] > d.max_tokens)
      return fail(KVQ_ERR_CAPACITY, "sequence %d: %d + %d tokens exceed max_tokens = %d", i, c->L[i], n_new[i],
                  d.max_tokens);
    any |= n_new[i] > 0;
  }
  if (!any) return ok();
  if (!K || !V) return fail(KVQ_ERR_ARG, "K and V must be device pointers");

  std::vector<int> seqs;
  std::vector<int32_t> L_new(d.batch), Lq_new(d.batch);
  bool fused = true;
  int64_t pages_needed = 0;
  for (int i = 0; i < d.batch; ++i) {
    L_new[i] = c->L[i] + n_new[i];
    Lq_new[i] = packed_len(c, i, L_new[i]);
    if (n_new[i] > 0) seqs.push_back(i);
    // a launch that both packs and fills the ring must not overwrite a slot
    // it still reads: safe when the tokens span at most the ring, or when
    // none of the tokens to pack sits in the ring
    if (n_new[i] > 0 && (int64_t)L_new[i] - c->Lq[i] > c->W && c->L[i] > c->Lq[i]) fused = false;
    if (c->paged)
      pages_needed += (Lq_new[i] + d.page_tokens - 1) / d.page_tokens - (int64_t)c->pages[i].size();
  }
  if (c->paged && pages_needed > (int64_t)c->free_pages.size())
    return fail(KVQ_ERR_CAPACITY, "the append needs %lld more pages, the pool has %zu free", (long long)pages_needed,
                c->free_pages.size());
  const auto classes = bit_classes(c, seqs);  // (no memory is asked for once anything has changed)
  for (int i = 0; c->paged && i < d.batch; ++i) c->pages[i].reserve((Lq_new[i] + d.page_tokens - 1) / d.page_tokens);
  {
    // a sequence's first packed group starts a fresh bound on its value
    // scales (after kvq_seq_release or kvq_cache_reset the old one is stale)
    kvq::WordReset r{};
    r.arena = c->arena;
    for (int i = 0; i < d.batch; ++i) {
      if (c->Lq[i] != 0 || Lq_new[i] == 0) continue;
      for (int h = 0; h < d.num_kv_heads; ++h) {
        r.off[r.n++] = c->head0[i] + (uint64_t)h * c->lay[i].stride + c->lay[i].vb;
        if (r.n == kvq::kTableSetMax) {
          const int e = kvq::launch_word_reset(r, stream);
          if (e) return hip_fail(e, "bound reset launch");
          r.n = 0;
        }
      }
    }
    const int e = kvq::launch_word_reset(r, stream);
    if (e) return hip_fail(e, "bound reset launch");
  }
  if (c->paged && pages_needed > 0) {
    // take the pages and write their block-table entries (ordered before the append launch)
    kvq::TableSet t{};
    t.table = const_cast<int32_t*>(c->pm.table);
    for (int i = 0; i < d.batch; ++i) {
      const int32_t want = (Lq_new[i] + d.page_tokens - 1) / d.page_tokens;
      while ((int32_t)c->pages[i].size() < want) {
        const int32_t pg = c->free_pages.back();
        c->free_pages.pop_back();
        t.idx[t.n] = i * c->pm.max_pages + (int32_t)c->pages[i].size();
        t.val[t.n] = pg;
        ++t.n;
        c->pages[i].push_back(pg);
        if (t.n == kvq::kTableSetMax) {
          const int e = kvq::launch_table_set(t, stream);
          if (e) return hip_fail(e, "block table launch");
          t.n = 0;
        }
      }
    }
    const int e = kvq::launch_table_set(t, stream);
    if (e) return hip_fail(e, "block table launch");
  }

  // fused: one launch packs groups and fills ring slots; otherwise pack
  // first, then fill the ring.
  const int phases = fused ? 1 : 2;
  for (int ph = 0; ph < phases; ++ph) {
    const bool quant = fused || ph == 0, copy = fused || ph == 1;
    for (auto& cls : classes) {
      kvq::AppendArgs a{};
      const HeadLayout& lay = c->lay[cls.second[0]];
      a.arena = c->arena;
      a.K = static_cast<const uint16_t*>(K);
      a.V = static_cast<const uint16_t*>(V);
      a.head_stride = lay.stride;
      a.kc = kvq::region_units(lay.kc); a.km = kvq::region_units(lay.km); a.vc = kvq::region_units(lay.vc);
      a.vm = kvq::region_units(lay.vm); a.tk = kvq::region_units(lay.tk); a.tv = kvq::region_units(lay.tv); a.vb = kvq::region_units(lay.vb);
      a.n_max = n_max; a.hkv = d.num_kv_heads; a.gk = d.key_group; a.gv = d.value_group; a.W = c->W;
      a.quantize = quant ? 1 : 0;
      a.pm = c->pm;
      int wg = 0, n = 0;
      for (int i : cls.second) {
        kvq::AppendSeq& s = a.seq[n++];
        s.head0 = c->head0[i];
        s.seq = i;
        s.L_old = c->L[i]; s.Lq_old = c->Lq[i]; s.L_new = L_new[i]; s.Lq_new = Lq_new[i];
        s.n_quant = (Lq_new[i] - c->Lq[i]) / d.key_group;
        const int32_t stay = L_new[i] - std::max(Lq_new[i], c->L[i]);
        s.n_copy = copy ? (stay + kvq::kCopyTokens - 1) / kvq::kCopyTokens : 0;
        s.n_query = rot && rot->q && ph == 0 ? (n_new[i] + kvq::kQueryTokens - 1) / kvq::kQueryTokens : 0;
        s.wg_begin = wg;
        wg += ((quant ? s.n_quant : 0) + s.n_copy + s.n_query) * d.num_kv_heads;
      }
      a.nseq = n;
      a.total_wg = wg;
      const int e = launch(a, rot, cls.first.first, cls.first.second, stream);
      if (e) return hip_fail(e, "append launch");
    }
  }
  for (int i = 0; i < d.batch; ++i) {
    c->L[i] = L_new[i];
    c->Lq[i] = Lq_new[i];
  }
  return ok();
}

}  // namespace kvq

extern "C" {

kvq_status kvq_append(kvq_cache* c, const void* K, const void* V, int32_t n_max, const int32_t* n_new,
                      void* stream) try {
  const auto packed = [](const kvq::AppendArgs& a, const kvq::RotaryArgs*, int bk, int bv, void* s) {
    return kvq::launch_append(a, bk, bv, s);
  };
  return kvq::append_tokens(c, K, V, n_max, n_new, nullptr, c && c->block ? c->block->append : packed, stream);
} catch (const std::bad_alloc&) {
  return no_memory();
}

size_t kvq_workspace_bytes(const kvq_cache* c) {
  if (!c) return 0;
  if (c->block) return c->block->bound(c, 1, -1, 0);
  return (size_t)c->d.batch * c->d.num_q_heads * (size_t)splits_bound(c) * kvq::kRecFloats * sizeof(float);
}

}  // extern "C"

// The split plan and the launches of decode, shared by the entry points below.
namespace {

// Query rows of a launch (see DecodeArgs): nqry queries per sequence in row
// groups of qpr queries, rows = qpr * (Hq / Hkv) rows per workgroup.
struct Rows {
  int nqry = 1, qpr = 1, nrg = 1, rows = 1;
  bool many = false;  // the many-row kernel (prefill_mfma.hip)
};

// Single-token decode: one row group of the kv head's query heads.  Chunk
// queries of the classes of decode_exact.hip: groups of 16 rows.  Of the others
// (32 rows in the chunk kernel for 1- and 2-bit classes, 16 for
// those and 4-bit classes, with value groups of 32 channels; 8, 5 or 4 in
// the decode kernel), the row group of whole queries with the smallest
// estimated time: ceil(nqry / qpr) passes over the kv head's cache at a
// per-pass cost that grows with the rows; the last group may repeat the last
// query in its spare rows, and a chunk kernel group of five heads leaves the
// rows past its 3 or 6 queries spare.
// Relative cost of one pass per row count: µs per row group of 131072-token
// K1V1 Llama-3.1-8B layers when a chunk launch takes several (4-row 18,
// 8-row 21, 16-row 30, 32-row 38; a launch's first pass costs 10-20 µs
// more).
int pass_cost(int rows) { return rows >= 32 ? 38 : rows >= 16 ? 30 : rows >= 8 ? 21 : rows >= 5 ? 19 : 18; }

Rows rows_for(const kvq_cache* c, bool matrix, int nqry, int bk, int bv) {
  const int gqh = c->d.num_q_heads / c->d.num_kv_heads;
  Rows r;
  r.rows = gqh;
  if (nqry <= 1) return r;
  r.nqry = nqry;
  if (!matrix) {  // one tile of 16 rows holds whole queries; the rest are spare
    r.rows = 16;
    r.qpr = 16 / gqh;
    r.nrg = (nqry + r.qpr - 1) / r.qpr;
    return r;
  }
  const bool rows16 = c->d.value_group == 32 && bk + bv <= 8;
  r.qpr = 1;  // one query per group (rows = gqh) unless a candidate is cheaper
  r.nrg = nqry;
  int best = -1;
  for (int rg : {32, 16, 8, 5, 4}) {
    if (rg >= 16 && !rows16) continue;
    if (rg == 32 && !kvq::chunk_rows32(bk, bv)) continue;
    // the decode kernel's row layouts hold whole sets of heads; the chunk
    // kernel's 16 or 32 rows take floor(rows / gqh) queries (five heads: 3
    // or 6) and leave the remaining rows spare
    if (rg < 16 && rg % gqh != 0) continue;
    const int qpr = rg / gqh, nrg = (nqry + qpr - 1) / qpr;
    const int cost = nrg * pass_cost(rg);
    if (best < 0 || cost < best) {
      best = cost;
      r.qpr = qpr;
      r.nrg = nrg;
      r.rows = rg;
    }
  }
  return r;  // 4 rows (1, 2 or 4 heads), 5 or 8 always qualify
}

struct SplitPlan {
  std::vector<int32_t> st, nq, ns, base;  // per sequence: split length, packed splits, all splits, first record
  std::vector<uint8_t> direct;            // per sequence: written by the split launch, not merged (empty: none)
  std::vector<uint8_t> many;              // per sequence of a windowed call: on the many-row kernel
  int64_t records = 0;   // what the launches write
  int64_t required = 0;  // what the caller's workspace has to hold
  int nqry = 1;
};

// Whether a class's chunk queries go to the many-row kernel, by (query, head)
// rows per kv head and, at 4-bit keys and values, by rows times tokens:
//   1- and 2-bit classes from 80 rows on: 80 rows of 4096 tokens (K2V2) take 24
//   us, 76 in 32-row groups 34; of 32768 tokens 50 and 64, but 64 rows 40;
//   K4V4 (which has 16-row groups of half the products per row) from 256 rows
//   and 3 * 2^20 rows x tokens on: 512 rows of 8192 tokens 51 against 62 us, of
//   4096 tokens 40 against 39, 256 rows of 1024 tokens 20 against 18;
//   8-bit classes, which have 8-row groups only, from 256 rows on: 28 against
//   37 us at 4096 tokens, 19 against 18 at 1024;
//   value groups of 64 and 128 channels (8-row groups at any width) from 80.
bool many_rows(const kvq_cache* c, int seq0, int nqry) {
  if (!c->matrix[seq0] || nqry <= 1) return false;
  const int64_t rows = (int64_t)nqry * (c->d.num_q_heads / c->d.num_kv_heads);
  const int bk = c->bk[seq0], bv = c->bv[seq0];
  if (bk + bv <= 4 || c->d.value_group != 32) return rows >= 80;
  if (bk + bv > 8) return rows >= 256;
  int64_t longest = 0;
  for (int i = 0; i < c->d.batch; ++i)
    if (c->bk[i] == bk && c->bv[i] == bv) longest = std::max<int64_t>(longest, c->L[i]);
  return rows >= 256 && rows * longest >= (int64_t)3 << 20;
}

// Splits of a class on the many-row kernel: the block count per split with the
// smallest estimated time.  One workgroup of eight waves fills a compute
// unit, so a launch takes rounds of one workgroup per unit; each costs its
// blocks and a fixed part, and more than one split writes and re-reads the
// records.  A block of 4- or 8-bit operands, which take two halves, has a time
// of its own.  Against forced splits (1 to 16; K1V1, K2V2, K4V4 and K8V8, 128 and
// 512 queries of four and eight heads, 512 to 16384 tokens) the plan is within
// 5% of the fastest; K2V2, 512 queries of four heads over 8192 tokens: 353 us in
// one split, 194 in two, 141 in three, 116 in four.
constexpr double kBlockUs = 1.33, kBlockUs2 = 1.65, kSplitUs = 10.2, kRecordUs = 2.1e-4;
int many_rows_blocks(const kvq_cache* c, const std::vector<int>& seqs, int nqry, int64_t max_records) {
  const double block_us = c->bk[seqs[0]] + c->bv[seqs[0]] <= 4 ? kBlockUs : kBlockUs2;
  const int gqh = c->d.num_q_heads / c->d.num_kv_heads;
  const int nrg = (nqry + 32 / gqh - 1) / (32 / gqh), nrw = (nrg + kvq::kPrefillWaves - 1) / kvq::kPrefillWaves;
  const int64_t bound = splits_bound(c), units = (int64_t)c->d.num_kv_heads * nrw, cus = target_workgroups(1);
  int64_t longest = 1;
  for (int i : seqs) longest = std::max<int64_t>(longest, (c->L[i] + 31) / 32);
  if (c->split_tokens > 0) {
    const int64_t bps = std::max<int64_t>(c->split_tokens / 32, (longest + bound - 1) / bound);
    int64_t records = 0;
    for (int i : seqs) records += ((c->L[i] + 31) / 32 + bps - 1) / bps;
    return (int)(records <= max_records ? bps : longest);
  }
  double best = 0.0;
  int64_t pick = longest;
  for (int64_t ns = 1; ns <= std::min<int64_t>(bound, 64); ++ns) {
    const int64_t bps = (longest + ns - 1) / ns;
    int64_t wgs = 0, records = 0;
    for (int i : seqs) {
      const int64_t n = ((c->L[i] + 31) / 32 + bps - 1) / bps;
      wgs += units * n;
      records += n > 1 ? n : 0;
    }
    if (records > max_records) break;
    const int64_t rounds = (wgs + cus - 1) / cus;
    const double t = rounds * (bps * block_us + kSplitUs) +
                     records * (double)nqry * c->d.num_q_heads * kRecordUs;
    if (ns == 1 || t < best) best = t, pick = bps;
  }
  return (int)pick;
}

// ws_bytes: the workspace at hand (the many-row kernel takes no more splits
// than fit it; one split needs none).
SplitPlan plan_splits(const kvq_cache* c, int nqry = 1, size_t ws_bytes = 0) {
  SplitPlan p;
  p.nqry = nqry;
  const int B = c->d.batch;
  p.st.assign(B, 0);
  std::map<std::pair<int, int>, std::vector<int>> classes;
  for (int i = 0; i < B; ++i) classes[{c->bk[i], c->bv[i]}].push_back(i);
  for (auto& cl : classes) {
    const bool matrix = c->matrix[cl.second[0]] != 0;
    const Rows r = rows_for(c, matrix, nqry, cl.first.first, cl.first.second);
    const int occ = nqry > 1 && matrix
                        ? kvq::matrix_decode_occupancy(cl.first.first, cl.first.second, c->d.key_group, r.rows)
                        : 0;
    const int32_t st = split_tokens_for(c, cl.second, nqry, r.nrg, occ);
    for (int i : cl.second) p.st[i] = st;
  }
  p.nq.resize(B);
  p.ns.resize(B);
  p.base.resize(B);
  for (int i = 0; i < B; ++i) {
    p.nq[i] = (c->Lq[i] + p.st[i] - 1) / p.st[i];
    p.ns[i] = p.nq[i] + (c->L[i] > c->Lq[i] ? 1 : 0);
    p.base[i] = (int32_t)p.records;
    p.records += p.ns[i];
  }
  p.required = p.records;
  if (nqry <= 1) return p;
  bool many = false;
  for (auto& cl : classes) many |= many_rows(c, cl.second[0], nqry);
  if (!many) return p;
  p.direct.assign(B, 0);
  // re-plan the many-row classes; the records of the others come first
  int64_t left = (int64_t)(ws_bytes / ((size_t)c->d.num_q_heads * nqry * kvq::kRecFloats * sizeof(float)));
  p.records = 0;
  for (int i = 0; i < B; ++i) {
    if (many_rows(c, i, nqry)) continue;
    p.base[i] = (int32_t)p.records;
    p.records += p.ns[i];
  }
  for (auto& cl : classes) {
    if (!many_rows(c, cl.second[0], nqry)) continue;
    const int bps = many_rows_blocks(c, cl.second, nqry, left - p.records);
    for (int i : cl.second) {
      p.nq[i] = bps;
      p.ns[i] = ((c->L[i] + 31) / 32 + bps - 1) / bps;
      p.direct[i] = p.ns[i] <= 1;
      p.base[i] = (int32_t)p.records;
      p.records += p.direct[i] ? 0 : p.ns[i];
    }
  }
  return p;
}

// Append inputs of a fused append + decode: the tokens [L_old[i], L[i]) of
// each sequence come from K/V rows and are written into the ring by the
// decode launch itself.
struct FusedAppend {
  const void* K;
  const void* V;
  int32_t n_max;
  const std::vector<int32_t>* L_old;
};

// The parts of a launch's arguments that follow from the cache and its rows.
void fill_args(kvq::DecodeArgs& a, const kvq_cache* c, int seq0, const Rows& r, const void* q, void* ws) {
  const kvq_cache_desc& d = c->d;
  const HeadLayout& lay = c->lay[seq0];
  a.arena = c->arena;
  a.q = static_cast<const uint16_t*>(q);
  a.ws = static_cast<float*>(ws);
  a.head_stride = lay.stride;
  a.kc = kvq::region_units(lay.kc); a.km = kvq::region_units(lay.km); a.vc = kvq::region_units(lay.vc);
  a.vm = kvq::region_units(lay.vm); a.tk = kvq::region_units(lay.tk); a.tv = kvq::region_units(lay.tv); a.vb = kvq::region_units(lay.vb);
  a.hq = d.num_q_heads; a.hkv = d.num_kv_heads; a.gk = d.key_group; a.gv = d.value_group; a.W = c->W;
  a.qscale = (float)(1.4426950408889634 / std::sqrt((double)d.head_dim));
  a.nqry = r.nqry; a.qpr = r.qpr; a.nrg = r.nrg; a.gqh = d.num_q_heads / d.num_kv_heads;
  // rows past qpr whole queries (a chunk kernel group of five heads) are
  // spare: row_x = kvq::kSpareRow marks them (a repeat of the last query)
  for (int g = 0; g < 32; ++g) {
    a.row_x[g] = g < r.qpr * a.gqh ? g / a.gqh : kvq::kSpareRow;
    a.row_off[g] = a.row_x[g] * d.num_q_heads + g % a.gqh;
  }
  a.pm = c->pm;
}

// The launch's sequences (one bit class) and their workgroups.
void fill_seqs(kvq::DecodeArgs& a, const kvq_cache* c, const std::vector<int>& seqs, const SplitPlan& p, const Rows& r) {
  const int row_wgs = r.many ? (r.nrg + kvq::kPrefillWaves - 1) / kvq::kPrefillWaves : r.nrg;
  int wg = 0, n = 0;
  for (int i : seqs) {
    kvq::DecodeSeq& s = a.seq[n++];
    s.head0 = c->head0[i];
    s.seq = i; s.L = s.L_old = c->L[i]; s.Lq = c->Lq[i];
    s.nq = p.nq[i]; s.nsplit = p.ns[i]; s.ws_base = p.base[i];
    s.wg_begin = wg;
    wg += p.ns[i] * c->d.num_kv_heads * row_wgs;
  }
  a.nseq = n;
  a.total_wg = wg;
}

// Whether the workspace fits `records` records of a plan's rows.
kvq_status check_workspace(const kvq_cache* c, int64_t records, int nqry, const void* ws, size_t ws_bytes) {
  const size_t need = (size_t)records * c->d.num_q_heads * nqry * kvq::kRecFloats * sizeof(float);
  if (need > 0 && !ws) return fail(KVQ_ERR_ARG, "workspace is NULL");
  if (ws_bytes < need) return fail(KVQ_ERR_CAPACITY, "workspace holds %zu bytes, this call needs %zu", ws_bytes, need);
  if (reinterpret_cast<uintptr_t>(ws) % 16 != 0) return fail(KVQ_ERR_ARG, "workspace must be 16-byte aligned");
  return KVQ_OK;
}

kvq_status run_partials(const kvq_cache* c, const SplitPlan& p, const void* q, void* ws, size_t ws_bytes,
                        void* stream, const FusedAppend* app = nullptr, float* out = nullptr) {
  const kvq_cache_desc& d = c->d;
  if (!q) return fail(KVQ_ERR_ARG, "q must be a device pointer");
  const kvq_status st = check_workspace(c, p.required, p.nqry, ws, ws_bytes);
  if (st != KVQ_OK) return st;
  std::vector<int> seqs;
  for (int i = 0; i < d.batch; ++i)
    if (c->L[i] > 0) seqs.push_back(i);
  for (auto& cls : bit_classes(c, seqs)) {
    kvq::DecodeArgs a{};
    Rows r = rows_for(c, c->matrix[cls.second[0]] != 0, p.nqry, cls.first.first, cls.first.second);
    if (many_rows(c, cls.second[0], p.nqry)) {
      r.many = true;
      r.rows = 32;
      r.qpr = 32 / (d.num_q_heads / d.num_kv_heads);
      r.nrg = (p.nqry + r.qpr - 1) / r.qpr;
      a.out = out;
    }
    fill_args(a, c, cls.second[0], r, q, ws);
    a.split_tokens = p.st[cls.second[0]];
    if (app) {
      a.K_new = static_cast<const uint16_t*>(app->K);
      a.V_new = static_cast<const uint16_t*>(app->V);
      a.n_max = app->n_max;
    }
    fill_seqs(a, c, cls.second, p, r);
    for (int k = 0; app && k < a.nseq; ++k) a.seq[k].L_old = (*app->L_old)[a.seq[k].seq];
    const int e = !c->matrix[cls.second[0]] ? kvq::launch_decode(a, cls.first.first, cls.first.second, r.rows, stream)
                  : r.rows >= 16 ? kvq::launch_chunk_matrix(a, cls.first.first, cls.first.second, r.rows, stream)
                                       : kvq::launch_decode_matrix(a, cls.first.first, cls.first.second, r.rows, stream);
    if (e) return hip_fail(e, "decode launch");
  }
  return KVQ_OK;
}

kvq_status run_merge(const kvq_cache* c, const SplitPlan& p, const void* ws, float* out, void* stream) {
  const kvq_cache_desc& d = c->d;
  if (!out) return fail(KVQ_ERR_ARG, "out must be a device pointer");
  if (p.records > 0 && !ws) return fail(KVQ_ERR_ARG, "workspace is NULL");
  for (int b = 0; b < d.batch; b += kvq::kMaxSeqPerLaunch) {
    kvq::MergeArgs m{};
    m.ws = static_cast<const float*>(ws);
    m.out = out;
    m.hq = d.num_q_heads * p.nqry;  // out [batch][nqry][Hq] = [batch][nqry * Hq]
    int n = 0;
    for (int i = b; i < std::min(d.batch, b + kvq::kMaxSeqPerLaunch); ++i) {
      if (!p.direct.empty() && p.direct[i]) continue;
      m.seq[n].seq = i; m.seq[n].nsplit = p.ns[i]; m.seq[n].ws_base = p.base[i];
      ++n;
    }
    m.nseq = n;
    const int e = kvq::launch_merge(m, stream);
    if (e) return hip_fail(e, "merge launch");
  }
  return KVQ_OK;
}

// ------------------------------------------------------------ windowed attention

// Fewest (query, head) rows per kv head for which the many-row kernel is considered
// (its 256-row workgroup is then a quarter full; with fewer it never won).
constexpr int kWindowManyFrom = 64;
constexpr double kWindowBlockUs2 = 2.0;   // a block of 4- or 8-bit operands with the values' low halves
constexpr double kWindowRecordUs = 5e-4;  // of one row and split, under 2048 rows

// Rows of a class's windowed launch: 16-row groups of whole queries, or row groups
// of 32 of the many-row kernel (the last group may repeat the last query).
Rows window_rows(const kvq_cache* c, int nqry, bool many) {
  const int gqh = c->d.num_q_heads / c->d.num_kv_heads;
  Rows r;
  r.nqry = nqry;
  r.many = many;
  r.rows = many ? 32 : 16;
  r.qpr = std::min(nqry, r.rows / gqh);
  r.nrg = (nqry + r.qpr - 1) / r.qpr;
  return r;
}

// Most packed key groups (many rows: blocks, the tail's too) that any workgroup
// of sequence i reads.
int32_t window_reach(const kvq_cache* c, int i, const Rows& r, int32_t window, int32_t sinks) {
  const int32_t seen0 = c->L[i] - r.nqry + 1, gsh = log2_exact(c->d.key_group);
  const int32_t step = r.qpr * (r.many ? kvq::kPrefillWaves : 1);  // queries per workgroup
  int32_t most = 0;
  for (int first = 0; first < r.nqry; first += step) {
    const int32_t seen_first = seen0 + first, seen_last = seen0 + std::min(first + step, r.nqry) - 1;
    int32_t n = kvq::window_groups(seen_first, seen_last, c->Lq[i], gsh, window, sinks).count;
    if (r.many) {
      const int32_t tail0 = sinks <= c->Lq[i] ? std::max(c->Lq[i], std::max(seen_first - window, 0)) / 32 : c->Lq[i] / 32;
      n = (n << (gsh - 5)) + std::max(0, (int32_t)(((int64_t)seen_last + 31) / 32) - tail0);
    }
    most = std::max(most, n);
  }
  return most;
}

// Most splits of a sequence in a windowed call, at any lengths.
int64_t window_splits(const kvq_cache* c, int nqry, int32_t window, int32_t sinks) {
  const int64_t gk = c->d.key_group, qpr = std::min(nqry, 32 / (c->d.num_q_heads / c->d.num_kv_heads));
  // a range of n tokens touches at most (n + gk - 2) / gk + 1 key groups
  const int64_t reach = std::min<int64_t>(c->cq / gk, (sinks + gk - 1) / gk + (window + qpr - 1 + gk - 2) / gk + 1);
  const int64_t per = c->split_tokens > 0 ? c->split_tokens / gk : kMinGroupsPerSplit;
  return std::min<int64_t>(kMaxSplits, (reach + per - 1) / per) + 1;
}

// Workgroups of a launch's row groups per sequence and split.
int64_t window_units(const kvq_cache* c, const Rows& r) {
  return (int64_t)c->d.num_kv_heads * (r.many ? (r.nrg + kvq::kPrefillWaves - 1) / kvq::kPrefillWaves : r.nrg);
}
bool window_many_possible(const kvq_cache* c, int seq0, int nqry) {
  return c->window[seq0] && (int64_t)nqry * (c->d.num_q_heads / c->d.num_kv_heads) >= kWindowManyFrom;
}

// Workgroups that a class of n sequences is split into at most: 8 rounds of one per
// compute unit, 16 for several sequences.  So many even out unequal lengths by
// themselves, and the records of the splits, which the workspace has to hold at any
// lengths, grow with them.  (Without a limit: 64 sequences of 100 to 9000 tokens, five
// queries, 12 rounds 198 us, 8 rounds 212; 32 of 500 to 8000, 64 queries, 356 us and
// 349, in a workspace of 2.2 GB and 0.28; one sequence takes 7 rounds at most.)
int64_t window_workgroups(int64_t n) { return (n > 1 ? 16 : 8) * target_workgroups(1); }

// Most splits of all sequences of a windowed call together, at any lengths.
int64_t window_records(const kvq_cache* c, int nqry, int32_t window, int32_t sinks) {
  const int64_t each = window_splits(c, nqry, window, sinks);
  if (c->split_tokens > 0) return c->d.batch * each;
  int64_t most = 0;
  for (const auto& cl : c->classes) {
    int64_t units = window_units(c, window_rows(c, nqry, false));
    if (window_many_possible(c, cl.first, nqry)) units = std::min(units, window_units(c, window_rows(c, nqry, true)));
    most += std::min<int64_t>(cl.second * each, window_workgroups(cl.second) / units);
  }
  return std::max<int64_t>(most, 1);
}

// Estimated time of a windowed launch of 16-row groups: workgroups, key blocks that a
// wave of the longest takes, rows to merge.  A compute unit holds two workgroups,
// but one already keeps its vector units near half busy, so each further one costs
// 0.85 of the first.  Splits are joined by a launch of their own.  Against forced
// splits (1 to 128 sequences of 8 kv heads, windows of 1024 to 16384 tokens, K2V2 to
// K8V8) the plan is within 8% of the fastest: 64 windows of 1024 tokens, K4V4, 31 us
// in one split each and 42 in two; 8 of 4096, K2V2, 23 in four, 26 in eight, 46 in
// one; 32 of 8192, K8V8 of five heads, 130 in one, 146 in two, 155 in six.
double window_us(int64_t wgs, int64_t blocks, int64_t merged_rows) {
  const int64_t cus = target_workgroups(1), rounds = (wgs + cus - 1) / cus;
  return 4.0 + (4.0 + 1.15 * (double)blocks) * (rounds > 1 ? 0.85 * (double)rounds : 1.0) +
         (merged_rows > 0 ? 5.0 + 3e-3 * (double)merged_rows : 0.0);
}
// Of one on the many-row kernel, which reads a block once for 256 rows: blocks of the
// longest workgroup, rows per kv head, records (rows times splits) and rows to merge
// (few of those take the merge of a workgroup per 32 channels).  4- or 8-bit
// operands: two halves.  The two estimates choose the kernel; against each alone (1,
// 4 and 16 sequences of four heads per kv head, 8 to 512 queries, windows of 512 and
// 4096, K2V2 and K4V4) within 10% of the better: one window of 512 tokens, K2V2, 256
// queries 24 us in tiles and 26, 512 queries 40 and 33; of 4096 tokens 32 queries 27
// and 30, 64 33 and 29, 512 134 and 77; 16 sequences of 4096, 16 queries 73 and 98, 32
// 135 and 102, 128 499 and 217.
double window_many_us(int64_t wgs, int64_t blocks, bool wide, int64_t head_rows, int64_t records, int64_t merged_rows) {
  const int64_t cus = target_workgroups(1);
  const double fill = 0.6 + 0.4 * (double)std::min<int64_t>(head_rows, 256) / 256;  // (waves without rows only unpack)
  return (double)((wgs + cus - 1) / cus) * ((double)blocks * fill * (wide ? kWindowBlockUs2 : kBlockUs) + kSplitUs) +
         (double)records * (merged_rows < 2048 ? kWindowRecordUs : kRecordUs);
}

// How a class's windowed launch is split: key groups (many rows: blocks) per split,
// and its estimated time.  reach: of each of its sequences.
struct WindowSplit {
  Rows r;
  std::vector<int32_t> reach;
  int64_t per = 0;
  double us = 0.0;
};
WindowSplit split_window(const kvq_cache* c, const std::vector<int>& seqs, int nqry, int32_t window, int32_t sinks, bool many,
                         int64_t bound) {
  WindowSplit w;
  w.r = window_rows(c, nqry, many);
  const int64_t units = window_units(c, w.r);
  const int64_t least = many ? 1 : kMinGroupsPerSplit, rows = (int64_t)nqry * c->d.num_q_heads;
  const int64_t most = window_workgroups((int64_t)seqs.size());
  const bool wide = c->bk[seqs[0]] + c->bv[seqs[0]] > 4;
  int64_t longest = 1;
  for (int i : seqs) {
    w.reach.push_back(window_reach(c, i, w.r, window, sinks));
    longest = std::max<int64_t>(longest, w.reach.back());
  }
  for (int64_t ns = 1; ns <= std::min<int64_t>(bound, 64); ++ns) {
    const int64_t n = std::max<int64_t>((longest + ns - 1) / ns, least);
    int64_t wgs = 0, records = 0, merged = 0;
    for (int32_t reach : w.reach) {
      const int64_t k = std::max<int64_t>(1, (reach + n - 1) / n);
      wgs += units * k;
      records += k > 1 ? k * rows : 0;
      merged += k > 1 ? rows : 0;
    }
    if (ns > 1 && wgs > most) break;
    const double t = many ? window_many_us(wgs, n, wide, rows / c->d.num_kv_heads, records, merged)
                          : window_us(wgs, (n + least - 1) / least * (c->d.key_group / 32), merged);
    if (ns == 1 || t < w.us) w.us = t, w.per = n;
    if (n == least) break;
  }
  return w;
}

// The split plan of a windowed call: the splits with the smallest estimated time,
// every sequence's of the same number of key groups (16-row groups: no fewer than
// one per wave; many rows: blocks, as for chunk queries).  The fp16 tail has a
// workgroup of its own where a compute unit is idle and the splits are merged anyway
// (one window of 1024 tokens, K2V2: the launch 8 us, 11 otherwise), else it belongs to
// the last split (64 of them: 34 us, 58 otherwise); a sequence of one split needs no
// merge.
SplitPlan plan_window(const kvq_cache* c, int nqry, int32_t window, int32_t sinks) {
  SplitPlan p;
  p.nqry = nqry;
  const int B = c->d.batch, gk = c->d.key_group;
  p.st.assign(B, 0);
  p.nq.assign(B, 0);
  p.ns.assign(B, 0);
  p.base.assign(B, 0);
  p.direct.assign(B, 0);
  p.many.assign(B, 0);
  const int64_t bound = window_splits(c, nqry, window, sinks);
  std::map<std::pair<int, int>, std::vector<int>> classes;
  for (int i = 0; i < B; ++i)
    if (c->L[i] > 0) classes[{c->bk[i], c->bv[i]}].push_back(i);
  for (auto& cl : classes) {
    const std::vector<int>& seqs = cl.second;
    WindowSplit w = split_window(c, seqs, nqry, window, sinks, false, bound);
    if (window_many_possible(c, seqs[0], nqry)) {
      WindowSplit other = split_window(c, seqs, nqry, window, sinks, true, bound);
      if (other.us < w.us) w = std::move(other);
    }
    const int64_t longest = *std::max_element(w.reach.begin(), w.reach.end());
    if (c->split_tokens > 0) w.per = c->split_tokens / (w.r.many ? 32 : gk);
    w.per = w.r.many ? std::max(w.per, (longest + bound - 1) / bound) : std::max(w.per, (longest + kMaxSplits - 1) / kMaxSplits);
    const int64_t units = (int64_t)c->d.num_kv_heads * w.r.nrg;
    int64_t wgs = 0, tails = 0;
    for (size_t k = 0; k < seqs.size(); ++k) {
      const int i = seqs[k];
      p.many[i] = w.r.many;
      p.ns[i] = (int32_t)std::max<int64_t>(1, (w.reach[k] + w.per - 1) / w.per);
      p.nq[i] = w.r.many ? (int32_t)w.per : (int32_t)((w.reach[k] + w.per - 1) / w.per);
      p.st[i] = w.r.many ? 0 : (int32_t)(w.per * gk);
      wgs += units * p.ns[i];
      if (p.nq[i] > 1 && c->L[i] > c->Lq[i]) tails += units;
    }
    const bool own_tails = !w.r.many && wgs + tails <= target_workgroups(1);
    for (int i : seqs) {
      if (own_tails && p.nq[i] > 1 && c->L[i] > c->Lq[i]) ++p.ns[i];
      p.direct[i] = p.ns[i] == 1;
      if (p.direct[i] && !w.r.many) p.required = 1;  // (a workspace is asked for whether or not the lengths leave it unused)
    }
  }
  for (int i = 0; i < B; ++i) {
    p.base[i] = (int32_t)p.records;
    p.records += p.direct[i] ? 0 : p.ns[i];
  }
  p.required = std::max(p.required, p.records);
  return p;
}

kvq_status run_window(const kvq_cache* c, const SplitPlan& p, const void* q, int32_t window, int32_t sinks, float* out,
                      void* ws, size_t ws_bytes, void* stream) {
  const kvq_status st = check_workspace(c, p.required, p.nqry, ws, ws_bytes);
  if (st != KVQ_OK) return st;
  std::vector<int> seqs;
  for (int i = 0; i < c->d.batch; ++i)
    if (c->L[i] > 0) seqs.push_back(i);
  for (auto& cls : bit_classes(c, seqs)) {
    kvq::DecodeArgs a{};
    const Rows r = window_rows(c, p.nqry, p.many[cls.second[0]] != 0);
    fill_args(a, c, cls.second[0], r, q, ws);
    a.split_tokens = p.st[cls.second[0]];
    a.window = window;
    a.sinks = sinks;
    a.out = out;
    fill_seqs(a, c, cls.second, p, r);
    const int e = r.many ? kvq::launch_window_rows(a, cls.first.first, cls.first.second, stream)
                         : kvq::launch_window(a, cls.first.first, cls.first.second, stream);
    if (e) return hip_fail(e, "windowed attention launch");
  }
  return KVQ_OK;
}

}  // namespace

extern "C" {

kvq_status kvq_decode_attention(const kvq_cache* c, const void* q, float* out, void* ws, size_t ws_bytes,
                                void* stream) try {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (!q || !out) return fail(KVQ_ERR_ARG, "q and out must be device pointers");
  if (c->block) return c->block->attend(c, q, 1, -1, 0, out, ws, ws_bytes, stream);
  const SplitPlan p = plan_splits(c);
  kvq_status st = run_partials(c, p, q, ws, ws_bytes, stream);
  if (st != KVQ_OK) return st;
  st = run_merge(c, p, ws, out, stream);
  if (st != KVQ_OK) return st;
  return ok();
} catch (const std::bad_alloc&) {
  return no_memory();
}

kvq_status kvq_decode_attention_noalloc(const kvq_cache* c, const void* q, float* out, void* stream) try {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (!q || !out) return fail(KVQ_ERR_ARG, "q and out must be device pointers");
  const SplitPlan p = c->block ? SplitPlan{} : plan_splits(c);
  const size_t need = c->block ? c->block->need(c, 1, -1, 0)
                               : (size_t)p.records * c->d.num_q_heads * kvq::kRecFloats * sizeof(float);
  if (need > kvq::kScratchBytes)
    return fail(KVQ_ERR_CAPACITY, "this decode needs %zu bytes of workspace, more than the %zu bytes of the "
                "library's scratch array; use kvq_decode_attention with a caller workspace", need, kvq::kScratchBytes);
  void* ws = nullptr;
  const int e = kvq::scratch_workspace(&ws);
  if (e) return hip_fail(e, "scratch array address");
  if (c->block) return c->block->attend(c, q, 1, -1, 0, out, ws, kvq::kScratchBytes, stream);
  kvq_status st = run_partials(c, p, q, ws, kvq::kScratchBytes, stream);
  if (st != KVQ_OK) return st;
  st = run_merge(c, p, ws, out, stream);
  if (st != KVQ_OK) return st;
  return ok();
} catch (const std::bad_alloc&) {
  return no_memory();
}

kvq_status kvq_append_decode(kvq_cache* c, const void* K, const void* V, int32_t n_max, const int32_t* n_new,
                             const void* q, float* out, void* ws, size_t ws_bytes, void* stream) try {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (!n_new) return fail(KVQ_ERR_ARG, "n_new is NULL");
  if (n_max < 0) return fail(KVQ_ERR_ARG, "n_max must be >= 0");
  if (!q || !out) return fail(KVQ_ERR_ARG, "q and out must be device pointers");
  const kvq_cache_desc& d = c->d;
  bool any = false, flush = false;
  for (int i = 0; i < d.batch; ++i) {
    if (n_new[i] < 0 || n_new[i] > n_max)
      return fail(KVQ_ERR_ARG, "sequence %d: n_new = %d outside [0, n_max = %d]", i, n_new[i], n_max);
    if ((int64_t)c->L[i] + n_new[i] > d.max_tokens)
      return fail(KVQ_ERR_CAPACITY, "sequence %d: %d + %d tokens exceed max_tokens = %d", i, c->L[i], n_new[i],
                  d.max_tokens);
    any |= n_new[i] > 0;
    flush |= packed_len(c, i, (int64_t)c->L[i] + n_new[i]) != c->Lq[i];
  }
  if (any && (!K || !V)) return fail(KVQ_ERR_ARG, "K and V must be device pointers");
  if (any && (reinterpret_cast<uintptr_t>(K) % 4 != 0 || reinterpret_cast<uintptr_t>(V) % 4 != 0))
    return fail(KVQ_ERR_ARG, "K and V must be 4-byte aligned");

  // plan with the lengths after the append; nothing is launched or changed
  // unless the workspace fits
  const std::vector<int32_t> L_old = c->L, Lq_old = c->Lq;
  const auto restore = [&] {
    c->L = L_old;
    c->Lq = Lq_old;
  };
  for (int i = 0; i < d.batch; ++i) {
    c->L[i] = L_old[i] + n_new[i];
    c->Lq[i] = packed_len(c, i, c->L[i]);
  }
  try {
    const SplitPlan p = c->block ? SplitPlan{} : plan_splits(c);
    const size_t need = c->block ? c->block->need(c, 1, -1, 0) : (size_t)p.records * d.num_q_heads * kvq::kRecFloats * sizeof(float);
    const char* bad = nullptr;
    kvq_status bad_st = KVQ_ERR_ARG;
    if (need > 0 && !ws) bad = "workspace is NULL";
    else if (ws_bytes < need) bad = "workspace too small for the lengths after the append", bad_st = KVQ_ERR_CAPACITY;
    else if (reinterpret_cast<uintptr_t>(ws) % 16 != 0) bad = "workspace must be 16-byte aligned";
    flush |= c->block != nullptr;  // (they have no fused step)
    if (bad || flush) restore();
    if (bad) return fail(bad_st, "%s (needs %zu bytes, has %zu)", bad, need, ws_bytes);
    if (flush) {  // a key group fills: the append kernel packs it, then a plain decode
      kvq_status st = kvq_append(c, K, V, n_max, n_new, stream);
      if (st != KVQ_OK) return st;
      return kvq_decode_attention(c, q, out, ws, ws_bytes, stream);
    }
    const FusedAppend app{K, V, n_max, &L_old};
    kvq_status st = run_partials(c, p, q, ws, ws_bytes, stream, any ? &app : nullptr);
    if (st != KVQ_OK) return st;
    st = run_merge(c, p, ws, out, stream);
    if (st != KVQ_OK) return st;
    return ok();
  } catch (const std::bad_alloc&) {  // (before the first launch, which is what stores the tokens)
    restore();
    throw;
  }
} catch (const std::bad_alloc&) {
  return no_memory();
}

kvq_status kvq_decode_partials(const kvq_cache* c, const void* q, void* ws, size_t ws_bytes, void* stream) try {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (c->block) return fail(KVQ_ERR_UNSUPPORTED, "a block-scaled cache has no split records");
  const kvq_status st = run_partials(c, plan_splits(c), q, ws, ws_bytes, stream);
  return st == KVQ_OK ? ok() : st;
} catch (const std::bad_alloc&) {
  return no_memory();
}

kvq_status kvq_decode_merge(const kvq_cache* c, const void* ws, float* out, void* stream) try {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (c->block) return fail(KVQ_ERR_UNSUPPORTED, "a block-scaled cache has no split records");
  const kvq_status st = run_merge(c, plan_splits(c), ws, out, stream);
  return st == KVQ_OK ? ok() : st;
} catch (const std::bad_alloc&) {
  return no_memory();
}

size_t kvq_chunk_workspace_bytes(const kvq_cache* c, int32_t n_q) {
  if (!c || n_q < 1 || n_q > KVQ_MAX_CHUNK) return 0;
  if (c->block) return c->block->bound(c, n_q, -1, 0);
  return kvq_workspace_bytes(c) * (size_t)n_q;
}

kvq_status kvq_chunk_attention(const kvq_cache* c, const void* q, int32_t n_q, float* out, void* ws,
                               size_t ws_bytes, void* stream) try {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (n_q < 1 || n_q > KVQ_MAX_CHUNK) return fail(KVQ_ERR_ARG, "n_q = %d outside [1, %d]", n_q, KVQ_MAX_CHUNK);
  if (!q || !out) return fail(KVQ_ERR_ARG, "q and out must be device pointers");
  for (int i = 0; i < c->d.batch; ++i)
    if (c->L[i] < n_q)
      return fail(KVQ_ERR_ARG, "sequence %d holds %d tokens, fewer than the %d chunk queries", i, c->L[i], n_q);
  if (c->block) return c->block->attend(c, q, n_q, -1, 0, out, ws, ws_bytes, stream);
  const SplitPlan p = plan_splits(c, n_q, ws_bytes);
  kvq_status st = run_partials(c, p, q, ws, ws_bytes, stream, nullptr, out);
  if (st != KVQ_OK) return st;
  st = run_merge(c, p, ws, out, stream);
  if (st != KVQ_OK) return st;
  return ok();
} catch (const std::bad_alloc&) {
  return no_memory();
}

size_t kvq_window_workspace_bytes(const kvq_cache* c, int32_t n_q, int32_t window, int32_t sinks) {
  if (!c || n_q < 1 || n_q > KVQ_MAX_CHUNK || window < 1 || sinks < 0) return 0;
  if (c->block) return c->block->bound(c, n_q, window, sinks);
  return (size_t)window_records(c, n_q, window, sinks) * c->d.num_q_heads * n_q * kvq::kRecFloats * sizeof(float);
}

kvq_status kvq_window_attention(const kvq_cache* c, const void* q, int32_t n_q, int32_t window, int32_t sinks,
                                float* out, void* ws, size_t ws_bytes, void* stream) try {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (n_q < 1 || n_q > KVQ_MAX_CHUNK) return fail(KVQ_ERR_ARG, "n_q = %d outside [1, %d]", n_q, KVQ_MAX_CHUNK);
  if (window < 1) return fail(KVQ_ERR_ARG, "window = %d must be at least 1", window);
  if (sinks < 0) return fail(KVQ_ERR_ARG, "sinks = %d must not be negative", sinks);
  if (!q || !out) return fail(KVQ_ERR_ARG, "q and out must be device pointers");
  int32_t longest = 1;
  for (int i = 0; i < c->d.batch; ++i) {
    if (n_q > 1 && c->L[i] < n_q)
      return fail(KVQ_ERR_ARG, "sequence %d holds %d tokens, fewer than the %d queries", i, c->L[i], n_q);
    longest = std::max(longest, c->L[i]);
  }
  window = std::min(window, longest);
  sinks = std::min(sinks, longest);
  if (c->block) return c->block->attend(c, q, n_q, window, sinks, out, ws, ws_bytes, stream);
  const SplitPlan p = plan_window(c, n_q, window, sinks);
  kvq_status st = run_window(c, p, q, window, sinks, out, ws, ws_bytes, stream);
  if (st != KVQ_OK) return st;
  st = run_merge(c, p, ws, out, stream);
  if (st != KVQ_OK) return st;
  return ok();
} catch (const std::bad_alloc&) {
  return no_memory();
}

kvq_status kvq_dequant(const kvq_cache* c, int32_t seq, int32_t tok0, int32_t ntok, float* K_out, float* V_out,
                       void* stream) {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (seq < 0 || seq >= c->d.batch) return fail(KVQ_ERR_ARG, "seq %d out of range", seq);
  if (tok0 < 0 || ntok < 0 || (int64_t)tok0 + ntok > c->L[seq])
    return fail(KVQ_ERR_ARG, "token range [%d, %lld) outside [0, %d)", tok0, (long long)tok0 + ntok, c->L[seq]);
  if (ntok == 0) return ok();
  if (!K_out || !V_out) return fail(KVQ_ERR_ARG, "outputs must be device pointers");
  const HeadLayout& lay = c->lay[seq];
  kvq::DequantArgs a{};
  a.arena = c->arena;
  a.head0 = c->head0[seq];
  a.seq = seq;
  a.pm = c->pm;
  a.K_out = K_out; a.V_out = V_out;
  a.head_stride = lay.stride;
  a.kc = kvq::region_units(lay.kc); a.km = kvq::region_units(lay.km); a.vc = kvq::region_units(lay.vc);
  a.vm = kvq::region_units(lay.vm); a.tk = kvq::region_units(lay.tk); a.tv = kvq::region_units(lay.tv);
  a.hkv = c->d.num_kv_heads; a.gk = c->d.key_group; a.gv = c->d.value_group; a.W = c->W;
  a.bk = c->block ? c->type_k : c->bk[seq]; a.bv = c->block ? c->type_v : c->bv[seq]; a.Lq = c->Lq[seq]; a.tok0 = tok0; a.ntok = ntok;
  const int e = c->block ? c->block->dequant(a, stream) : kvq::launch_dequant(a, stream);
  if (e) return hip_fail(e, "dequant launch");
  return ok();
}

size_t kvq_export_bytes(const kvq_cache* c, int32_t seq, int32_t h) {
  if (!c || seq < 0 || seq >= c->d.batch || h < 0 || h >= c->d.num_kv_heads) return 0;
  const size_t Lq = c->Lq[seq], tail = c->L[seq] - c->Lq[seq], D = kvq::kHeadDim;
  if (c->block) return Lq * 2 * D + Lq / c->d.key_group * 2 * sizeof(float) + tail * D * 2 * 2;
  return Lq * 16 * c->bk[seq] + Lq / c->d.key_group * 2 * D * 2 + Lq * 16 * c->bv[seq] +
         Lq * (D / c->d.value_group) * 4 + tail * D * 2 * 2;
}

kvq_status kvq_export(const kvq_cache* c, int32_t seq, int32_t h, void* dst, size_t bytes, void* stream) {
  const size_t need = kvq_export_bytes(c, seq, h);
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (seq < 0 || seq >= c->d.batch || h < 0 || h >= c->d.num_kv_heads)
    return fail(KVQ_ERR_ARG, "(seq %d, kv head %d) out of range", seq, h);
  if (bytes < need) return fail(KVQ_ERR_CAPACITY, "destination holds %zu bytes, the image has %zu", bytes, need);
  if (need == 0) return ok();
  if (!dst) return fail(KVQ_ERR_ARG, "destination is NULL");
  const HeadLayout& lay = c->lay[seq];
  const size_t Lq = c->Lq[seq], tail = c->L[seq] - c->Lq[seq], D = kvq::kHeadDim;
  kvq::ExportArgs x{};
  x.arena = c->arena;
  x.head0 = c->head0[seq];
  x.head_stride = lay.stride;
  x.kc_out = static_cast<uint8_t*>(dst);
  x.km_out = x.kc_out + Lq * 16 * c->bk[seq];
  x.vc_out = x.km_out + Lq / c->d.key_group * 2 * D * 2;
  x.vm_out = x.vc_out + Lq * 16 * c->bv[seq];
  x.tk_out = x.vm_out + Lq * (D / c->d.value_group) * 4;
  if (c->block) {  // key codes, scales, value codes, scales, then the tails
    x.vc_out = x.km_out + Lq / c->d.key_group * sizeof(float);
    x.vm_out = x.vc_out + Lq * D;
    x.tk_out = x.vm_out + Lq / c->d.key_group * sizeof(float);
    x.bk = c->type_k;
    x.bv = c->type_v;
  }
  x.tv_out = x.tk_out + tail * D * 2;
  x.kc = kvq::region_units(lay.kc); x.km = kvq::region_units(lay.km); x.vc = kvq::region_units(lay.vc);
  x.vm = kvq::region_units(lay.vm); x.tk = kvq::region_units(lay.tk); x.tv = kvq::region_units(lay.tv);
  if (!c->block) x.bk = c->bk[seq], x.bv = c->bv[seq];
  x.gk = c->d.key_group; x.gv = c->d.value_group; x.W = c->W;
  x.Lq = (int32_t)Lq; x.ntail = (int32_t)tail; x.seq = seq; x.h = h;
  x.pm = c->pm;
  const int e = c->block ? c->block->export_image(x, stream) : kvq::launch_export(x, stream);
  if (e) return hip_fail(e, "export launch");
  return ok();
}

kvq_status kvq_check(const kvq_cache* c, void* stream) {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  hipError_t e = hipStreamSynchronize(static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "stream synchronize");
  uint32_t flag = 0;
  e = hipMemcpy(&flag, c->arena, sizeof flag, hipMemcpyDeviceToHost);
  if (e != hipSuccess) return hip_fail(e, "read error flag");
  if (flag == (uint32_t)KVQ_ERR_RANGE)
    return fail(KVQ_ERR_RANGE, "an append met a non-finite input or a group range beyond the fp16 scale");
  return ok();
}

kvq_status kvq_set_split_tokens(kvq_cache* c, int32_t tokens) {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (tokens < 0 || (tokens > 0 && tokens % c->d.key_group != 0))
    return fail(KVQ_ERR_ARG, "split tokens %d must be 0 or a positive multiple of key_group %d", tokens,
                c->d.key_group);
  if (tokens > 0 && (c->cq + tokens - 1) / tokens > kMaxSplits)
    return fail(KVQ_ERR_ARG, "split tokens %d would give more than %d splits at capacity", tokens, kMaxSplits);
  c->split_tokens = tokens;
  return ok();
}

// ------------------------------------------------------------------ DGAP

size_t dgap_workspace_bytes(int32_t batch, int32_t vocab, int32_t k) {
  if (batch < 1 || k < DGAP_MIN_K || k > DGAP_MAX_K || vocab < k || vocab > (1 << 24)) return 0;
  const int64_t nchunk = (vocab + kvq::kDgapChunk - 1) / kvq::kDgapChunk;
  if (nchunk * k > kvq::kDgapMaxCandidates) return 0;
  const uint64_t stats = ((uint64_t)batch * nchunk * 4 * sizeof(float) + kvq::kAlign - 1) / kvq::kAlign * kvq::kAlign;
  return (size_t)(stats + (uint64_t)batch * nchunk * k * sizeof(uint64_t));
}

size_t dgap_info_floats(int32_t k) { return (size_t)kvq::kDgapInfoHead + 2 * (size_t)(k > 0 ? k : 0); }

kvq_status dgap_restore(const dgap_params* p, float* logits, int32_t batch, void* ws, size_t ws_bytes, float* info,
                        void* stream) {
  if (!p) return fail(KVQ_ERR_ARG, "params is NULL");
  if (batch < 1) return fail(KVQ_ERR_ARG, "batch must be >= 1 (got %d)", batch);
  if (p->k < DGAP_MIN_K || p->k > DGAP_MAX_K)
    return fail(KVQ_ERR_ARG, "k = %d outside [%d, %d]", p->k, DGAP_MIN_K, DGAP_MAX_K);
  if (p->vocab < p->k) return fail(KVQ_ERR_ARG, "vocab %d smaller than k %d", p->vocab, p->k);
  if (p->hidden_det < 1 || p->hidden_det > DGAP_MAX_HIDDEN || p->hidden_corr < 1 || p->hidden_corr > DGAP_MAX_HIDDEN)
    return fail(KVQ_ERR_ARG, "hidden sizes (%d, %d) outside [1, %d]", p->hidden_det, p->hidden_corr, DGAP_MAX_HIDDEN);
  if (!(p->tau == p->tau)) return fail(KVQ_ERR_ARG, "tau is NaN");
  if (!p->det_w1 || !p->det_b1 || !p->det_w2 || !p->corr_w1 || !p->corr_b1 || !p->corr_w2)
    return fail(KVQ_ERR_ARG, "a weight pointer is NULL");
  if (!logits) return fail(KVQ_ERR_ARG, "logits is NULL");
  const size_t need = dgap_workspace_bytes(batch, p->vocab, p->k);
  if (need == 0)
    return fail(KVQ_ERR_UNSUPPORTED, "vocab %d with k %d: at most 2^24 logits and %d window candidates per row",
                p->vocab, p->k, kvq::kDgapMaxCandidates);
  if (!ws) return fail(KVQ_ERR_ARG, "workspace is NULL");
  if (ws_bytes < need) return fail(KVQ_ERR_CAPACITY, "workspace holds %zu bytes, this call needs %zu", ws_bytes, need);
  if (reinterpret_cast<uintptr_t>(ws) % 16 != 0) return fail(KVQ_ERR_ARG, "workspace must be 16-byte aligned");
  kvq::DgapArgs a{};
  a.logits = logits;
  a.info = info;
  a.vocab = p->vocab;
  a.k = p->k;
  a.nchunk = (p->vocab + kvq::kDgapChunk - 1) / kvq::kDgapChunk;
  a.hidden_det = p->hidden_det;
  a.hidden_corr = p->hidden_corr;
  a.tau = p->tau;
  a.det_b2 = p->det_b2;
  a.corr_b2 = p->corr_b2;
  a.det_w1 = p->det_w1; a.det_b1 = p->det_b1; a.det_w2 = p->det_w2;
  a.corr_w1 = p->corr_w1; a.corr_b1 = p->corr_b1; a.corr_w2 = p->corr_w2;
  const uint64_t stats = ((uint64_t)batch * a.nchunk * 4 * sizeof(float) + kvq::kAlign - 1) / kvq::kAlign * kvq::kAlign;
  a.ws_stats = static_cast<float*>(ws);
  a.ws_cand = reinterpret_cast<uint64_t*>(static_cast<uint8_t*>(ws) + stats);
  const int e = kvq::launch_dgap(a, batch, stream);
  if (e) return hip_fail(e, "dgap launch");
  return ok();
}

// ------------------------------------------------------------------ sampling

size_t dgap_sample_workspace_bytes(int32_t batch, int32_t vocab) {
  if (batch < 1 || vocab < 1 || vocab > (1 << 24)) return 0;
  return (size_t)batch * sample_row_bytes(vocab);
}

kvq_status dgap_sample(const dgap_sampling* p, int32_t* tokens, float* logprobs, void* ws, size_t ws_bytes,
                       void* stream) {
  if (!p) return fail(KVQ_ERR_ARG, "parameters are NULL");
  kvq_status st = check_rows(p->logits, p->type, p->row_stride, p->batch, p->vocab, "batch");
  if (st != KVQ_OK) return st;
  if (!p->uniform || !tokens) return fail(KVQ_ERR_ARG, "uniform and tokens must be device pointers");
  st = check_scratch(ws, ws_bytes, dgap_sample_workspace_bytes(p->batch, p->vocab));
  if (st != KVQ_OK) return st;
  kvq::SampleArgs a{};
  a.logits = p->logits;
  a.temperature = p->temperature; a.top_k = p->top_k; a.top_p = p->top_p; a.min_p = p->min_p; a.uniform = p->uniform;
  a.tokens = tokens;
  a.logprobs = logprobs;
  a.ws = static_cast<uint8_t*>(ws);
  a.row_stride = p->row_stride;
  a.row_bytes = sample_row_bytes(p->vocab);
  a.batch = p->batch; a.vocab = p->vocab;
  a.ngroup = (p->vocab + kvq::kSampleGroup - 1) / kvq::kSampleGroup;
  if ((p->batch < kSampleRows && p->vocab > kSampleSmall) || p->vocab > kvq::kSampleNarrow) {
    // workgroups for every compute unit, of 2048 logits at least
    int64_t chunk = 8192;
    while (chunk > kvq::kSampleChunk && p->batch * ((p->vocab + chunk - 1) / chunk) < target_workgroups(1)) chunk /= 2;
    a.chunk = (int32_t)chunk;
    a.nchunk = (int32_t)((p->vocab + chunk - 1) / chunk);
  }
  // the sum of all weights stays below 2^63; 45: a bin 51 octaves below the
  // largest weight holds none
  a.unit = std::min(45, 62 - log2_exact(p->vocab));
  const int e = kvq::launch_sample(a, p->type, stream);
  if (e) return hip_fail(e, "sampling launch");
  return ok();
}

// ------------------------------------------------------------------ teacher loss

size_t dgap_distill_workspace_bytes(int32_t rows, int32_t vocab) {
  if (rows < 1 || vocab < 1 || vocab > (1 << 24)) return 0;
  return (size_t)rows * (8 + 8 * (size_t)((vocab + kvq::kDistillChunk - 1) / kvq::kDistillChunk));
}

kvq_status dgap_distill(const dgap_distillation* p, float* loss, float* lse, void* grad, int64_t grad_row_stride,
                        const float* grad_loss, void* ws, size_t ws_bytes, void* stream) {
  kvq::DistillArgs a{};
  kvq_status st = distill_args(a, p, grad, grad_row_stride, grad_loss, false);
  if (st != KVQ_OK) return st;
  if (!loss) return fail(KVQ_ERR_ARG, "loss must be a device pointer");
  st = check_scratch(ws, ws_bytes, dgap_distill_workspace_bytes(p->rows, p->vocab));
  if (st != KVQ_OK) return st;
  a.loss = loss;
  a.lse = lse;
  a.row_sum = static_cast<float*>(ws);
  a.ws = a.row_sum + 2 * (size_t)p->rows;
  const int e = kvq::launch_distill(a, p->type, stream);
  if (e) return hip_fail(e, "teacher loss launch");
  return ok();
}

kvq_status dgap_distill_backward(const dgap_distillation* p, const float* lse, const float* grad_loss, void* grad,
                                 int64_t grad_row_stride, void* stream) {
  kvq::DistillArgs a{};
  const kvq_status st = distill_args(a, p, grad, grad_row_stride, grad_loss, true);
  if (st != KVQ_OK) return st;
  if (!lse) return fail(KVQ_ERR_ARG, "lse must be a device pointer");
  a.lse = const_cast<float*>(lse);
  const int e = kvq::launch_distill(a, p->type, stream);
  if (e) return hip_fail(e, "teacher loss gradient launch");
  return ok();
}

const char* kvq_last_error(void) { return kvq::last_error(); }

kvq_status kvq_read_probe(const void* src, size_t bytes, uint32_t* sink, void* stream) {
  if (!src || !sink) return fail(KVQ_ERR_ARG, "src and sink must be device pointers");
  if (bytes % 16 != 0 || reinterpret_cast<uintptr_t>(src) % 16 != 0)
    return fail(KVQ_ERR_ARG, "src must be 16-byte aligned and bytes a multiple of 16");
  const int e = kvq::launch_read_probe(src, bytes, sink, stream);
  if (e) return hip_fail(e, "read probe launch");
  return ok();
}

size_t kvq_read_probe_sink_bytes(void) { return (size_t)kvq::read_probe_blocks() * sizeof(uint32_t); }

const char* kvq_version(void) { return "kvq 0.1.0 gfx950"; }

}  // extern "C"
