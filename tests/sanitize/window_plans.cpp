// Split plans of windowed calls over random caches and lengths (host code alone, under
// AddressSanitizer and UBSan): what a call needs never exceeds the workspace that it is
// said to need at any lengths, and that workspace does not grow with the batch.
// "window plans ok" on success.
#include "../../paper_2607_16248_amd/csrc/kvq_api.cpp"

#include <cstdio>
#include <random>

static int g_fail = 0;
#define EXPECT(cond)                                                       \
  do {                                                                     \
    if (!(cond)) {                                                         \
      std::fprintf(stderr, "FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); \
      ++g_fail;                                                            \
    }                                                                      \
  } while (0)

static void* const kArena = reinterpret_cast<void*>((uintptr_t)1 << 40);  // never dereferenced here

struct Cache {
  std::vector<uint8_t> bk, bv;
  kvq_cache_desc d{};
  kvq_cache* c = nullptr;
  Cache(std::vector<uint8_t> k, std::vector<uint8_t> v, int hq, int hkv, int maxt, int gk, int gv, int R) : bk(std::move(k)), bv(std::move(v)) {
    d.batch = (int)bk.size(); d.num_q_heads = hq; d.num_kv_heads = hkv; d.head_dim = 128; d.max_tokens = maxt;
    d.key_group = gk; d.value_group = gv; d.fp16_window = R; d.bits_k = bk.data(); d.bits_v = bv.data();
    EXPECT(kvq_cache_init(&c, &d, kArena, kvq_cache_bytes(&d)) == KVQ_OK);
  }
  ~Cache() { kvq_cache_destroy(c); }
  void length(int i, int L) {
    c->L[i] = L;
    c->Lq[i] = quantized_len(L, d);
  }
};

int main() {
  std::mt19937 g(7);
  auto pick = [&](std::vector<int> v) { return v[g() % v.size()]; };
  int split = 0;
  for (int it = 0; it < 4000; ++it) {
    const int B = pick({1, 1, 2, 3, 4, 7, 16, 32, 70}), hkv = pick({1, 2, 8, 8, 16}), gqh = pick({1, 2, 4, 5, 8});
    const int gk = pick({32, 32, 64, 128}), maxt = pick({600, 2048, 8192, 32768, 131072, 524288}), kinds = pick({1, 1, 2, 4});
    std::vector<uint8_t> bk(B), bv(B);
    for (int i = 0; i < B; ++i) bk[i] = (uint8_t)(1 << (i % kinds)), bv[i] = (uint8_t)(it % 2 ? 2 : bk[i]);
    Cache x(bk, bv, hkv * gqh, hkv, maxt, gk, pick({32, 32, 64, 16}), pick({0, 32, 130}));
    const int nq = pick({1, 1, 2, 5, 16, 33, 64, 128, 200, 511, 1000, 1024});
    if (nq > maxt) continue;
    const int window = pick({1, 64, 500, 1024, 4096, 32768, 1 << 30}), sinks = pick({0, 4, 100, 4096, 1 << 30});
    const int shape = pick({0, 1, 2});  // all full, ragged, one long one among short ones
    int longest = 1;
    for (int i = 0; i < B; ++i) {
      const int L = shape == 0 || (shape == 2 && i == B / 2) ? maxt : shape == 1 ? nq + (int)(g() % (uint32_t)(maxt - nq + 1)) : nq;
      x.length(i, nq == 1 && g() % 5 == 0 ? 0 : L);
      longest = std::max(longest, x.c->L[i]);
    }
    if (it % 7 == 0) EXPECT(kvq_set_split_tokens(x.c, std::max(gk, (maxt / 400 + gk - 1) / gk * gk)) == KVQ_OK);
    const SplitPlan p = plan_window(x.c, nq, std::min(window, longest), std::min(sinks, longest));
    const size_t row = (size_t)hkv * gqh * nq * kvq::kRecFloats * sizeof(float);
    EXPECT((size_t)p.required * row <= kvq_window_workspace_bytes(x.c, nq, window, sinks));
    EXPECT(p.required >= p.records);
    int64_t end = 0;
    for (int i = 0; i < B; ++i) {
      if (p.direct[i] || p.ns[i] == 0) continue;
      EXPECT(p.base[i] == end);
      end += p.ns[i];
      split += p.ns[i] > 1;
    }
    EXPECT(end == p.records);
  }
  EXPECT(split > 1000);
  // a chunk of 1024 queries of 32 heads: 17.3 MB of records a split, whatever the batch
  for (int B : {1, 2, 16, 64})
    for (int window : {4096, 1 << 30}) {
      Cache x(std::vector<uint8_t>(B, 2), std::vector<uint8_t>(B, 2), 32, 8, 131072, 32, 32, 128);
      EXPECT(kvq_window_workspace_bytes(x.c, 1024, window, 4) <= (B == 1 ? (size_t)300 << 20 : (size_t)600 << 20));
      EXPECT(kvq_window_workspace_bytes(x.c, 1, window, 4) <= (size_t)40 << 20);
    }
  if (g_fail) return 1;
  std::printf("window plans ok\n");
  return 0;
}
