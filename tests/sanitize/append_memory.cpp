// Appends of packed and block-scaled caches without host memory, under AddressSanitizer
// and UBSan: whichever allocation of a call fails, it returns a status with lengths and
// pages as they were, and the call works afterwards; so do the attention calls.  (An
// append_decode that consists of two calls may end between them.)  "append memory ok" on success.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>
#include <vector>

#include "kvq.h"

static long g_left = -1;  // allocations that still succeed; -1: all
void* operator new(size_t n) {
  if (g_left >= 0 && g_left-- == 0) {
    g_left = 0;
    throw std::bad_alloc();
  }
  if (void* p = std::malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

static int g_fail = 0;
#define EXPECT(cond)                                                       \
  do {                                                                     \
    if (!(cond)) {                                                         \
      std::fprintf(stderr, "FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); \
      ++g_fail;                                                            \
    }                                                                      \
  } while (0)

constexpr int B = 5, hkv = 2, gqh = 4, maxt = 600;

struct State {
  std::vector<int64_t> v;
  explicit State(const kvq_cache* c) {
    for (int i = 0; i < B; ++i) v.push_back(kvq_seq_len(c, i)), v.push_back((int64_t)kvq_export_bytes(c, i, 0));
    v.push_back(kvq_free_pages(c));
  }
};

// f fails after 0, 1, ... allocations, and changes nothing, until it does not
template <class F>
static int until_it_works(const kvq_cache* c, F f) {
  const State before(c);
  for (long n = 0; n < 1000; ++n) {
    g_left = n;
    const kvq_status st = f();
    g_left = -1;
    if (st == KVQ_OK) return (int)n;
    EXPECT(st == KVQ_ERR_CAPACITY);
    EXPECT(State(c).v == before.v);
  }
  EXPECT(!"works with all the memory it wants");
  return 0;
}

static int calls(kvq_cache* c, bool block) {
  int failed = 0;
  std::vector<uint16_t> x((size_t)B * maxt * (gqh + 2) * hkv * 128), q((size_t)B * 40 * gqh * hkv * 128);
  std::vector<float> table((size_t)maxt * 64), out((size_t)B * 40 * gqh * hkv * 128);
  const size_t bytes = kvq_chunk_workspace_bytes(c, 40);
  void* ws = std::aligned_alloc(256, (bytes + 255) / 256 * 256);
  std::vector<int32_t> n = {300, 1, 40, 150, 41}, one(B, 1);
  failed += until_it_works(c, [&] { return kvq_append(c, x.data(), x.data(), 300, n.data(), nullptr); });
  kvq_rotary r{};
  r.q = x.data(); r.k = r.v = x.data();
  r.q_stride = r.k_stride = r.v_stride = (gqh + 2) * hkv * 128;
  r.cos_table = r.sin_table = table.data();
  r.table_rows = maxt;
  r.rotary_dim = 128;
  std::vector<uint16_t> turned((size_t)B * 50 * gqh * hkv * 128);
  n = {50, 0, 40, 3, 1};
  failed += until_it_works(c, [&] { return kvq_append_rotary(c, &r, 50, n.data(), turned.data(), nullptr); });
  // steps: one in which no group fills is one launch that stores the tokens; the others (and
  // a block-scaled cache's) are an append and a decode, of which the second may fail alone
  for (int step = 0; step < 40; ++step) {
    const State before(c);
    for (long k = 0; k < 1000; ++k) {
      g_left = k;
      const kvq_status st = kvq_append_decode(c, x.data(), x.data(), 1, one.data(), q.data(), out.data(), ws, bytes, nullptr);
      g_left = -1;
      const bool appended = State(c).v != before.v;
      for (int i = 0; i < B; ++i) EXPECT(kvq_seq_len(c, i) == before.v[2 * i] + (appended ? 1 : 0));
      if (st == KVQ_OK) EXPECT(appended);
      if (st != KVQ_OK) EXPECT(st == KVQ_ERR_CAPACITY);
      if (st != KVQ_OK && appended) {
        bool filled = block;
        for (int i = 0; i < B; ++i) filled |= before.v[2 * i] + 1 >= 52 && (before.v[2 * i] + 1 - 20) % 32 == 0;
        EXPECT(filled);
        EXPECT(kvq_decode_attention(c, q.data(), out.data(), ws, bytes, nullptr) == KVQ_OK);
      }
      if (appended) break;
      ++failed;
    }
  }
  failed += until_it_works(c, [&] { return kvq_decode_attention(c, q.data(), out.data(), ws, bytes, nullptr); });
  failed += until_it_works(c, [&] { return kvq_chunk_attention(c, q.data(), 40, out.data(), ws, bytes, nullptr); });
  if (block) failed += until_it_works(c, [&] { return kvq_window_attention(c, q.data(), 40, 64, 4, out.data(), ws, bytes, nullptr); });
  std::free(ws);
  return failed;
}

int main() {
  int failed = 0;
  for (int page : {0, 128}) {
    const std::vector<uint8_t> bits(B, 4);
    kvq_cache_desc d{B, gqh * hkv, hkv, 128, maxt, 32, 32, 20, bits.data(), bits.data(), page, 0};
    kvq_block_desc b{B, gqh * hkv, hkv, 128, maxt, 32, 20, KVQ_I8, KVQ_E4M3, page, 0, 0};
    for (int block = 0; block < 2; ++block) {
      const size_t bytes = block ? kvq_block_cache_bytes(&b) : kvq_cache_bytes(&d);
      void* arena = std::aligned_alloc(256, (bytes + 255) / 256 * 256);
      std::memset(arena, 0, bytes);
      kvq_cache* c = nullptr;
      for (long left = 0; !c && left < 1000; ++left) {
        g_left = left;
        const kvq_status st = block ? kvq_block_cache_init(&c, &b, arena, bytes) : kvq_cache_init(&c, &d, arena, bytes);
        g_left = -1;
        EXPECT(c ? st == KVQ_OK : st == KVQ_ERR_CAPACITY);
        failed += !c;
      }
      failed += calls(c, block != 0);
      kvq_cache_destroy(c);
      std::free(arena);
    }
  }
  EXPECT(failed > 500);
  if (g_fail) return 1;
  std::printf("append memory ok\n");
  return 0;
}
