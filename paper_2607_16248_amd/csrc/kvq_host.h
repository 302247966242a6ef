// Host-side pieces shared by the sources of the C ABI: the cache handle, status
// and error helpers, and the append that every entry point ends in.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <utility>
#include <vector>

#include "dgap.h"
#include "kvq.h"
#include "kvq_internal.h"

namespace kvq {

// Launches the append kernels of a call; rot: the call's rotation, or null.
using AppendLaunch = int (*)(const AppendArgs& a, const RotaryArgs* rot, int bk, int bv, void* stream);

// What the calls do for a block-scaled cache (kvq_block.cpp) in place of the
// packed classes' kernels.  need: workspace bytes of a call at the current
// lengths; bound: at any lengths.  window < 0: no window.
struct BlockCalls {
  AppendLaunch append;
  size_t (*bound)(const kvq_cache* c, int32_t n_q, int32_t window, int32_t sinks);
  size_t (*need)(const kvq_cache* c, int32_t n_q, int32_t window, int32_t sinks);
  kvq_status (*attend)(const kvq_cache* c, const void* q, int32_t n_q, int32_t window, int32_t sinks, float* out,
                       void* ws, size_t ws_bytes, void* stream);
  int (*dequant)(const DequantArgs& a, void* stream);
  int (*export_image)(const ExportArgs& a, void* stream);
};

constexpr int kMaxSplits = 512;  // packed splits per sequence and kv head

kvq_status fail(kvq_status s, const char* fmt, ...);
kvq_status no_memory();
kvq_status ok();
kvq_status hip_fail(int e, const char* what);
const char* last_error();
int64_t target_workgroups(int per_cu);
int log2_exact(int v);
// Rows of logits that a call reads whole.
kvq_status check_rows(const void* logits, int type, int64_t row_stride, int rows, int vocab, const char* what);

int64_t packed_capacity(const kvq_cache_desc* d);
int32_t quantized_len(int64_t L, const kvq_cache_desc& d);
// A descriptor's checks, the arena it needs and a handle over it; block: a
// block-scaled cache's (bits_k and bits_v hold 8, value_group 128).
kvq_status check_desc(const kvq_cache_desc* d);
size_t arena_bytes(const kvq_cache_desc* d, bool block);
kvq_status init_cache(kvq_cache** out, const kvq_cache_desc* d, void* arena, size_t arena_bytes, bool block);

// kvq_append's checks and launches.  K, V: input rows as the launch reads them.
// rot: the call's rotation (its query workgroups are in the launch's grid), or null.
kvq_status append_tokens(kvq_cache* c, const void* K, const void* V, int32_t n_max, const int32_t* n_new,
                         const RotaryArgs* rot, AppendLaunch launch, void* stream);

}  // namespace kvq

struct kvq_cache {
  kvq_cache_desc d{};
  std::vector<uint8_t> bk, bv;
  uint8_t* arena = nullptr;
  size_t arena_bytes = 0;
  int64_t cq = 0;   // most tokens ever packed per sequence
  int32_t W = 0;    // ring slots per head
  std::vector<uint64_t> head0;
  std::vector<kvq::HeadLayout> lay;
  std::vector<int32_t> L, Lq;
  std::vector<uint8_t> matrix;  // 1: the kernels of decode_mfma.hip (else decode_exact.hip)
  std::vector<uint8_t> window;  // 1: the many-row kernel serves its windowed queries
  std::vector<std::pair<int, int>> classes;  // of equal key and value bits: the first sequence, how many there are
  std::vector<int> occupancy;    // resident decode workgroups per compute unit, per sequence's kernel
  int32_t split_tokens = 0;
  // paged layout: block table on the device (pm.table), page lists and the
  // free pool on the host
  bool paged = false;
  kvq::PageMap pm{};
  std::vector<std::vector<int32_t>> pages;  // per sequence: pool page of each logical page
  std::vector<int32_t> free_pages;           // taken from the back
  // block-scaled caches: their kernels (null: the packed classes'), element types
  const kvq::BlockCalls* block = nullptr;
  int32_t type_k = 0, type_v = 0;
};

namespace kvq {
// Packed tokens of sequence i when it holds L: what is packed stays packed
// (kvq_truncate drops tokens, not groups).
inline int32_t packed_len(const kvq_cache* c, int i, int64_t L) {
  const int32_t n = quantized_len(L, c->d);
  return n > c->Lq[i] ? n : c->Lq[i];
}
}  // namespace kvq
