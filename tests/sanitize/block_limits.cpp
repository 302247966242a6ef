// Plans of block-scaled attention at their limits: forced splits of one block under large
// batches and chunks (millions of parts), the longest caches.  Every call runs, does all
// work once (block_stub.cpp) and fits the workspace that it is said to need.  "block
// limits ok" on success.
#include <algorithm>
#include <cstdio>
#include <cstring>

// (buffers do not exist: no merge over them)
#include "kvq_internal.h"
namespace kvq {
int merge_of_no_buffers(const MergeArgs&, void*) { return 0; }
}
#define launch_merge merge_of_no_buffers
#include "../../paper_2607_16248_amd/csrc/kvq_block.cpp"
#undef launch_merge

extern bool g_touch;
extern int64_t g_parts;

static int g_fail = 0;
#define EXPECT(cond)                                                       \
  do {                                                                     \
    if (!(cond)) {                                                         \
      std::fprintf(stderr, "FAILED %s:%d: %s (%s)\n", __FILE__, __LINE__, #cond, kvq_last_error()); \
      ++g_fail;                                                            \
    }                                                                      \
  } while (0)

static void* const kFake = reinterpret_cast<void*>((uintptr_t)1 << 40);  // never dereferenced

static void attend(int B, int gqh, int hkv, int maxt, int block, int split, int nq) {
  kvq_block_desc d{B, gqh * hkv, hkv, 128, maxt, block, 0, KVQ_I8, KVQ_E4M3, 0, 0, 0};
  kvq_cache* c = nullptr;
  EXPECT(kvq_block_cache_init(&c, &d, kFake, kvq_block_cache_bytes(&d)) == KVQ_OK);
  for (int i = 0; i < B; ++i) {
    c->L[i] = maxt - i;
    c->Lq[i] = kvq::quantized_len(c->L[i], c->d);
  }
  EXPECT(kvq_set_split_tokens(c, split) == KVQ_OK);
  float* out = static_cast<float*>(kFake);
  if (nq == 1) EXPECT(kvq_decode_attention(c, kFake, out, kFake, kvq_workspace_bytes(c), nullptr) == KVQ_OK);
  EXPECT(kvq_chunk_attention(c, kFake, nq, out, kFake, kvq_chunk_workspace_bytes(c, nq), nullptr) == KVQ_OK);
  EXPECT(kvq_window_attention(c, kFake, nq, 5000, 64, out, kFake, kvq_window_workspace_bytes(c, nq, 5000, 64), nullptr) == KVQ_OK);
  kvq_cache_destroy(c);
}

int main() {
  g_touch = false;
  attend(70, 8, 16, 8192, 32, 32, 1024);  // 5.9 million parts of a block
  attend(64, 8, 32, 8192, 32, 32, 1024);
  attend(33, 1, 64, 16384, 32, 32, 90);
  attend(64, 4, 64, 16384, 32, 32, 1);
  attend(4, 8, 8, 1 << 20, 32, 0, 1024);
  attend(1, 8, 2, 9000000, 128, 0, 1);
  attend(1, 8, 2, 9000000, 128, 0, 300);
  EXPECT(g_parts > 10000000);
  if (g_fail) return 1;
  std::printf("block limits ok\n");
  return 0;
}
