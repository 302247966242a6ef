// C ABI of the rotated append (include/kvq.h): argument checks; the bookkeeping and
// the launches are kvq_append's.
#include <stdint.h>

#include <new>

#include "kvq.h"
#include "kvq_host.h"
#include "kvq_internal.h"

using kvq::fail;

extern "C" kvq_status kvq_append_rotary(kvq_cache* c, const kvq_rotary* r, int32_t n_max, const int32_t* n_new,
                                        void* q_out, void* stream) try {
  if (!c) return fail(KVQ_ERR_ARG, "cache is NULL");
  if (!r) return fail(KVQ_ERR_ARG, "parameters are NULL");
  if (!n_new) return fail(KVQ_ERR_ARG, "n_new is NULL");
  if (n_max < 0) return fail(KVQ_ERR_ARG, "n_max must be >= 0");
  bool any = false;
  for (int i = 0; i < c->d.batch; ++i) any |= n_new[i] > 0;
  if (r->type != KVQ_F16 && r->type != KVQ_BF16) return fail(KVQ_ERR_ARG, "type %d is none of kvq_type", r->type);
  if (r->rotary_dim < 16 || r->rotary_dim > kvq::kHeadDim || r->rotary_dim % 16 != 0)
    return fail(KVQ_ERR_ARG, "rotary_dim %d; must be a multiple of 16 up to %d", r->rotary_dim, kvq::kHeadDim);
  if (r->adjacent_pairs != 0 && r->adjacent_pairs != 1)
    return fail(KVQ_ERR_ARG, "adjacent_pairs %d; must be 0 or 1", r->adjacent_pairs);
  if (r->table_rows < 1 || r->table_rows > (int64_t)1 << 31)
    return fail(KVQ_ERR_ARG, "table_rows %lld outside [1, 2^31]", (long long)r->table_rows);
  if ((r->q == nullptr) != (q_out == nullptr)) return fail(KVQ_ERR_ARG, "q and q_out go together");
  const int64_t row = (int64_t)c->d.num_kv_heads * kvq::kHeadDim, q_row = (int64_t)c->d.num_q_heads * kvq::kHeadDim;
  if (r->k_stride < row || r->v_stride < row || (r->q && r->q_stride < q_row))
    return fail(KVQ_ERR_ARG, "strides (%lld, %lld, %lld) smaller than a token's rows", (long long)r->q_stride,
                (long long)r->k_stride, (long long)r->v_stride);
  const int64_t far = (int64_t)1 << 40;  // (offsets of any row stay far inside 64 bits)
  if (r->k_stride > far || r->v_stride > far || r->q_stride > far) return fail(KVQ_ERR_ARG, "strides above 2^40");
  if (any) {
    if (!r->k || !r->v) return fail(KVQ_ERR_ARG, "k and v must be device pointers");
    if (!r->cos_table || !r->sin_table) return fail(KVQ_ERR_ARG, "the tables must be device pointers");
  }
  if ((reinterpret_cast<uintptr_t>(r->k) | reinterpret_cast<uintptr_t>(r->v) | reinterpret_cast<uintptr_t>(r->q)) % 2 != 0)
    return fail(KVQ_ERR_ARG, "rows must be aligned to their type");
  if ((reinterpret_cast<uintptr_t>(r->cos_table) | reinterpret_cast<uintptr_t>(r->sin_table) |
       reinterpret_cast<uintptr_t>(r->positions) | reinterpret_cast<uintptr_t>(q_out)) % 4 != 0)
    return fail(KVQ_ERR_ARG, "tables, positions and q_out must be 4-byte aligned");
  for (int i = 0; !r->positions && i < c->d.batch; ++i)
    if (n_new[i] > 0 && (int64_t)c->L[i] + n_new[i] > r->table_rows)
      return fail(KVQ_ERR_ARG, "sequence %d: places up to %lld, the tables have %lld rows", i,
                  (long long)c->L[i] + n_new[i] - 1, (long long)r->table_rows);
  kvq::RotaryArgs a{};
  a.q = static_cast<const uint16_t*>(r->q);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.cos_ = r->cos_table;
  a.sin_ = r->sin_table;
  a.position = r->positions;
  a.q_stride = r->q_stride; a.k_stride = r->k_stride; a.v_stride = r->v_stride;
  a.rows = r->table_rows;
  a.rot = r->rotary_dim; a.pairs = r->adjacent_pairs; a.bf16 = r->type == KVQ_BF16;
  a.gqh = c->d.num_q_heads / c->d.num_kv_heads;
  const uintptr_t at = reinterpret_cast<uintptr_t>(r->k) | reinterpret_cast<uintptr_t>(r->v) | reinterpret_cast<uintptr_t>(r->q);
  const int64_t step = r->k_stride | r->v_stride | (r->q ? r->q_stride : 0);
  a.aligned = at % 16 == 0 && step % 8 == 0;
  return kvq::append_tokens(c, r->k, r->v, n_max, n_new, &a, c->block ? c->block->append : kvq::launch_append_rotary, stream);
} catch (const std::bad_alloc&) {
  return kvq::no_memory();
}
