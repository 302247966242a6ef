// The attention calls of the C interface without host memory, under AddressSanitizer and
// UBSan: whichever allocation of a call fails, it returns a status, and the next call
// works.  "host memory ok" on success.
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

// f fails after 0, 1, ... allocations until it does not
template <class F>
static int until_it_works(F f) {
  for (long n = 0; n < 1000; ++n) {
    g_left = n;
    const kvq_status st = f();
    g_left = -1;
    if (st == KVQ_OK) return (int)n;
    EXPECT(st == KVQ_ERR_CAPACITY);
  }
  EXPECT(!"works with all the memory it wants");
  return 0;
}

int main() {
  constexpr int B = 70, hq = 8, hkv = 2, maxt = 200, nq = 40;
  std::vector<uint8_t> bk(B), bv(B);
  for (int i = 0; i < B; ++i) bk[i] = bv[i] = (uint8_t)(1 << i % 4);
  kvq_cache_desc d{};
  d.batch = B; d.num_q_heads = hq; d.num_kv_heads = hkv; d.head_dim = 128; d.max_tokens = maxt; d.key_group = 32;
  d.value_group = 32; d.fp16_window = 20; d.bits_k = bk.data(); d.bits_v = bv.data();
  void* arena = std::aligned_alloc(256, (kvq_cache_bytes(&d) + 255) / 256 * 256);
  kvq_cache* c = nullptr;
  EXPECT(kvq_cache_init(&c, &d, arena, kvq_cache_bytes(&d)) == KVQ_OK);
  std::vector<uint16_t> kv((size_t)B * maxt * hkv * 128), q((size_t)B * nq * hq * 128);
  std::vector<float> out((size_t)B * nq * hq * 128);
  const std::vector<int32_t> n(B, 150);
  EXPECT(kvq_append(c, kv.data(), kv.data(), maxt, n.data(), nullptr) == KVQ_OK);
  const size_t bytes = kvq_chunk_workspace_bytes(c, nq);
  EXPECT(kvq_window_workspace_bytes(c, nq, 64, 4) <= bytes);
  void* ws = std::aligned_alloc(256, (bytes + 255) / 256 * 256);
  int failed = 0;
  failed += until_it_works([&] { return kvq_window_attention(c, q.data(), 1, 64, 4, out.data(), ws, bytes, nullptr); });
  failed += until_it_works([&] { return kvq_window_attention(c, q.data(), nq, 64, 4, out.data(), ws, bytes, nullptr); });
  failed += until_it_works([&] { return kvq_chunk_attention(c, q.data(), nq, out.data(), ws, bytes, nullptr); });
  failed += until_it_works([&] { return kvq_decode_attention(c, q.data(), out.data(), ws, bytes, nullptr); });
  failed += until_it_works([&] { return kvq_decode_partials(c, q.data(), ws, bytes, nullptr); });
  failed += until_it_works([&] { return kvq_decode_merge(c, ws, out.data(), nullptr); });
  EXPECT(failed > 50);
  const size_t want = kvq_window_workspace_bytes(c, nq, 64, 4);
  for (long left = 0; left < 1000; ++left) {  // 0 or the size
    g_left = left;
    const size_t got = kvq_window_workspace_bytes(c, nq, 64, 4);
    g_left = -1;
    EXPECT(got == 0 || got == want);
    if (got == want) break;
  }
  g_left = 0;  // refusals have a status without a message
  EXPECT(kvq_window_attention(c, q.data(), 0, 64, 4, out.data(), ws, bytes, nullptr) == KVQ_ERR_ARG);
  g_left = -1;
  kvq_cache_destroy(c);
  std::free(ws);
  std::free(arena);
  if (g_fail) return 1;
  std::printf("host memory ok\n");
  return 0;
}
