// Block-scaled caches, rotated appends and truncation under AddressSanitizer and UBSan
// (host code alone): plans over random caches and lengths do all work once
// (block_stub.cpp) and fit the workspace that a call is said to need; random runs of
// appends, truncations, releases and reads on caches with real buffers stay inside
// them; refusals change nothing.  "block plans ok" on success.
#include <cstdio>
#include <cstring>
#include <algorithm>
#include <random>

// (plans are also made over buffers that do not exist: the merge's stand-in is called
// where they do)
#include "kvq_internal.h"
namespace kvq {
int merge_of_real_buffers(const MergeArgs& a, void* stream);
}
#define launch_merge merge_of_real_buffers
#include "../../paper_2607_16248_amd/csrc/kvq_block.cpp"
#undef launch_merge

extern bool g_touch;
extern int64_t g_parts;
extern int g_tile_launches, g_row_launches;

int kvq::merge_of_real_buffers(const MergeArgs& a, void* stream) { return g_touch ? launch_merge(a, stream) : 0; }

static int g_fail = 0;
#define EXPECT(cond)                                                       \
  do {                                                                     \
    if (!(cond)) {                                                         \
      std::fprintf(stderr, "FAILED %s:%d: %s (%s)\n", __FILE__, __LINE__, #cond, kvq_last_error()); \
      ++g_fail;                                                            \
    }                                                                      \
  } while (0)

static std::mt19937 g(11);
static int pick(std::vector<int> v) { return v[g() % v.size()]; }
static void* const kFake = reinterpret_cast<void*>((uintptr_t)1 << 40);  // never dereferenced

static kvq_block_desc desc(int B, int gqh, int hkv, int maxt, int block, int R, int page = 0, int pages = 0) {
  return {B, gqh * hkv, hkv, 128, maxt, block, R, (int)(g() % 2), (int)(g() % 2), page, pages, 0};
}

static void plans() {
  g_touch = false;
  for (int it = 0; it < 2500; ++it) {
    const int B = pick({1, 1, 2, 3, 7, 16, 33, 70}), hkv = pick({1, 2, 8, 8, 16}), gqh = pick({1, 2, 4, 5, 8});
    const int block = pick({32, 64, 128}), maxt = pick({300, 2048, 8192, 32768, 131072}), R = pick({0, 32, 130, 1000});
    kvq_block_desc d = desc(B, gqh, hkv, maxt, block, R, pick({0, 0, 256}));
    kvq_cache* c = nullptr;
    EXPECT(kvq_block_cache_init(&c, &d, kFake, kvq_block_cache_bytes(&d)) == KVQ_OK);
    const int nq = pick({1, 1, 1, 2, 3, 5, 8, 16, 33, 64, 100, 256, 511, 1024});
    if (nq <= maxt) {
      const int shape = pick({0, 1, 2, 3});  // all full, ragged, one long one among short ones, short
      for (int i = 0; i < B; ++i) {
        const int most = shape == 3 ? std::min(maxt, nq + 200) : maxt;
        int L = shape == 0 || (shape == 2 && i == B / 2) ? maxt : shape != 2 ? nq + (int)(g() % (uint32_t)(most - nq + 1)) : nq;
        if (nq == 1 && g() % 6 == 0) L = 0;
        c->L[i] = L;
        c->Lq[i] = kvq::quantized_len(L, c->d);
        if (g() % 4 == 0) c->L[i] -= (int)(g() % (uint32_t)std::max(1, std::min(c->L[i] - c->Lq[i], c->L[i] - nq) + 1));  // truncated
        if (c->L[i] < 0) c->L[i] = 0;
      }
      if (it % 6 == 0) EXPECT(kvq_set_split_tokens(c, std::max(block, (maxt / pick({3, 50, 400}) + block - 1) / block * block)) == KVQ_OK);
      const int window = pick({1, 40, 500, 4096, 1 << 30}), sinks = pick({0, 4, 100, 1 << 30});
      float* out = static_cast<float*>(kFake);
      if (nq == 1) EXPECT(kvq_decode_attention(c, kFake, out, kFake, kvq_workspace_bytes(c), nullptr) == KVQ_OK);
      EXPECT(kvq_chunk_attention(c, kFake, nq, out, kFake, kvq_chunk_workspace_bytes(c, nq), nullptr) == KVQ_OK ||
             (nq == 1 && *std::min_element(c->L.begin(), c->L.end()) < 1));
      EXPECT(kvq_window_attention(c, kFake, nq, window, sinks, out, kFake, kvq_window_workspace_bytes(c, nq, window, sinks), nullptr) == KVQ_OK);
    }
    kvq_cache_destroy(c);
  }
  // the workspace does not grow with the batch: a split of 1024 queries of 32 heads is 17.3 MB
  for (int B : {1, 16, 64}) {
    kvq_block_desc d = desc(B, 4, 8, 131072, 64, 128);
    kvq_cache* c = nullptr;
    EXPECT(kvq_block_cache_init(&c, &d, kFake, kvq_block_cache_bytes(&d)) == KVQ_OK);
    EXPECT(kvq_chunk_workspace_bytes(c, 1024) <= (size_t)(8 + 3 * B) * 18 << 20);
    EXPECT(kvq_workspace_bytes(c) <= (size_t)(80 + 3 * B) * 17 << 10);
    kvq_cache_destroy(c);
  }
  g_touch = true;
}

struct Real {
  std::vector<uint8_t> buf;
  uint8_t* at;
  explicit Real(size_t n) : buf(n + 256) { at = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(buf.data()) + 255) / 256 * 256); }
};

// The packed classes are appended to as well (with a handle of kvq_cache_init).
static void runs(bool block) {
  for (int it = 0; it < 60; ++it) {
    const int B = pick({1, 2, 3}), hkv = pick({1, 2}), gqh = pick({1, 2, 4, 5}), G = pick({32, 64, 128}), R = pick({0, 5, 40, 130});
    const int maxt = pick({50, 300, 700}), page = pick({0, 128, 256}), pages = page ? pick({0, 3}) : 0;
    kvq_block_desc bd = desc(B, gqh, hkv, maxt, G, R, page, pages);
    std::vector<uint8_t> bits(B, (uint8_t)(1 << pick({0, 1, 2, 3})));
    kvq_cache_desc d{B, gqh * hkv, hkv, 128, maxt, G, 32, R, bits.data(), bits.data(), page, pages};
    const size_t bytes = block ? kvq_block_cache_bytes(&bd) : kvq_cache_bytes(&d);
    EXPECT(bytes > 0);
    Real arena(bytes);
    kvq_cache* c = nullptr;
    EXPECT((block ? kvq_block_cache_init(&c, &bd, arena.at, bytes) : kvq_cache_init(&c, &d, arena.at, bytes)) == KVQ_OK);
    for (int step = 0; step < 14; ++step) {
      const int n_max = pick({1, 1, 2, 7, 33, 150}), rot = pick({16, 32, 64, 96, 128}), rows = 1 + (int)(g() % 800);
      std::vector<int32_t> n(B), positions((size_t)B * n_max, 0);
      for (int i = 0; i < B; ++i) n[i] = (int)(g() % (uint32_t)(n_max + 1));
      const int width = (gqh + 2) * hkv * 128 + pick({0, 8, 24}), qs = pick({0, 1});
      std::vector<uint16_t> x((size_t)B * n_max * width), q_out((size_t)B * n_max * gqh * hkv * 128);
      std::vector<float> table((size_t)rows * (rot / 2));
      kvq_rotary r{};
      r.q = qs ? x.data() : nullptr;
      r.k = x.data() + (size_t)gqh * hkv * 128;
      r.v = x.data() + (size_t)(gqh + 1) * hkv * 128;
      r.q_stride = r.k_stride = r.v_stride = width;
      r.cos_table = r.sin_table = table.data();
      r.positions = g() % 2 ? positions.data() : nullptr;
      r.table_rows = rows;
      r.type = (int)(g() % 2);
      r.rotary_dim = rot;
      // (the last row's end: rows of q, k and v lie side by side)
      const std::vector<int32_t> before = c->L;
      bool fits = true, known = true;
      for (int i = 0; i < B; ++i) {
        fits &= before[i] + n[i] <= maxt;
        known &= n[i] == 0 || r.positions || before[i] + n[i] <= rows;
      }
      const kvq_status st = kvq_append_rotary(c, &r, n_max, n.data(), qs ? q_out.data() : nullptr, nullptr);
      EXPECT(st == KVQ_OK || st == KVQ_ERR_CAPACITY || (!known && st == KVQ_ERR_ARG));
      if (!known || !fits) EXPECT(st != KVQ_OK);
      for (int i = 0; i < B; ++i) EXPECT(c->L[i] == before[i] + (st == KVQ_OK ? n[i] : 0) && c->Lq[i] <= c->L[i] && c->L[i] - c->Lq[i] < R + G);
      if (g() % 3 == 0) {  // drop some of the newest
        std::vector<int32_t> lens(B);
        for (int i = 0; i < B; ++i) lens[i] = c->Lq[i] + (int)(g() % (uint32_t)(c->L[i] - c->Lq[i] + 1));
        EXPECT(kvq_truncate(c, lens.data()) == KVQ_OK);
        for (int i = 0; i < B; ++i) EXPECT(c->L[i] == lens[i]);
        const std::vector<int32_t> held = c->L;
        lens[0] = c->L[0] + 1;
        EXPECT(kvq_truncate(c, lens.data()) == KVQ_ERR_ARG && c->L == held);
        lens[0] = c->Lq[0] - 1;
        EXPECT(kvq_truncate(c, lens.data()) == (c->Lq[0] ? KVQ_ERR_STATE : KVQ_ERR_ARG) && c->L == held);
      }
      if (g() % 9 == 0) EXPECT(kvq_seq_release(c, (int)(g() % (uint32_t)B)) == KVQ_OK);
      if (!block) {  // a fused step after a truncation packs no group twice
        std::vector<uint16_t> kv((size_t)B * hkv * 128), q((size_t)B * gqh * hkv * 128);
        std::vector<float> out((size_t)B * gqh * hkv * 128);
        std::vector<int32_t> one(B, 0);
        for (int i = 0; i < B; ++i) one[i] = c->L[i] < maxt;
        Real ws(kvq_workspace_bytes(c));
        const kvq_status s2 = kvq_append_decode(c, kv.data(), kv.data(), 1, one.data(), q.data(), out.data(), ws.at, kvq_workspace_bytes(c), nullptr);
        EXPECT(s2 == KVQ_OK || s2 == KVQ_ERR_CAPACITY);
        continue;
      }
      const int32_t least = *std::min_element(c->L.begin(), c->L.end());
      for (int nq : {1, pick({2, 5, 17, 40})}) {
        std::vector<uint16_t> q((size_t)B * nq * gqh * hkv * 128);
        std::vector<float> out((size_t)B * nq * gqh * hkv * 128);
        Real ws(kvq_chunk_workspace_bytes(c, nq)), ww(kvq_window_workspace_bytes(c, nq, 50, 4));
        if (nq == 1) EXPECT(kvq_decode_attention(c, q.data(), out.data(), ws.at, kvq_workspace_bytes(c), nullptr) == KVQ_OK);
        if (least >= nq) {
          EXPECT(kvq_chunk_attention(c, q.data(), nq, out.data(), ws.at, kvq_chunk_workspace_bytes(c, nq), nullptr) == KVQ_OK);
          EXPECT(kvq_window_attention(c, q.data(), nq, 50, 4, out.data(), ww.at, kvq_window_workspace_bytes(c, nq, 50, 4), nullptr) == KVQ_OK);
        }
      }
      const int seq = (int)(g() % (uint32_t)B), h = (int)(g() % (uint32_t)hkv);
      std::vector<uint8_t> image(kvq_export_bytes(c, seq, h));
      EXPECT(kvq_export(c, seq, h, image.data(), image.size(), nullptr) == KVQ_OK);
      if (c->L[seq] > 0) {
        const int t0 = (int)(g() % (uint32_t)c->L[seq]), nt = 1 + (int)(g() % (uint32_t)(c->L[seq] - t0));
        std::vector<float> k((size_t)nt * hkv * 128), v(k.size());
        EXPECT(kvq_dequant(c, seq, t0, nt, k.data(), v.data(), nullptr) == KVQ_OK);
      }
      EXPECT(kvq_decode_partials(c, image.data(), nullptr, 0, nullptr) == KVQ_ERR_UNSUPPORTED);
    }
    kvq_cache_destroy(c);
  }
}

int main() {
  plans();
  runs(true);
  runs(false);
  EXPECT(g_parts > 100000 && g_tile_launches > 1000 && g_row_launches > 500);
  if (g_fail) return 1;
  std::printf("block plans ok, %lld parts\n", (long long)g_parts);
  return 0;
}
