// C ABI of the adjusted logits (include/dgap.h): argument checks and the launch.
#include <stdint.h>

#include "dgap.h"
#include "kvq_host.h"
#include "kvq_internal.h"

using kvq::fail;

extern "C" kvq_status dgap_adjust(const dgap_adjustment* p, void* out, int64_t out_row_stride, void* stream) {
  if (!p) return fail(KVQ_ERR_ARG, "parameters are NULL");
  const kvq_status st = kvq::check_rows(p->logits, p->type, p->row_stride, p->batch, p->vocab, "batch");
  if (st != KVQ_OK) return st;
  const int size = p->type == DGAP_F32 ? 4 : 2;
  if (!out) return fail(KVQ_ERR_ARG, "out must be a device pointer");
  if (reinterpret_cast<uintptr_t>(out) % size != 0) return fail(KVQ_ERR_ARG, "out must be aligned to its type");
  if (out_row_stride < p->vocab)
    return fail(KVQ_ERR_ARG, "out_row_stride %lld smaller than vocab %d", (long long)out_row_stride, p->vocab);
  if (out == p->logits && out_row_stride != p->row_stride)
    return fail(KVQ_ERR_ARG, "an output in the logits' place needs their row stride");
  if (p->history < 0 || p->history > 1 << 24) return fail(KVQ_ERR_ARG, "history = %d outside [0, 2^24]", p->history);
  if (p->biases < 0 || p->biases > DGAP_MAX_BIASES)
    return fail(KVQ_ERR_ARG, "biases = %d outside [0, %d]", p->biases, DGAP_MAX_BIASES);
  if (p->biases > 0 && (!p->bias_token || !p->bias))
    return fail(KVQ_ERR_ARG, "bias_token and bias must be device pointers");
  if (p->history > 0 && !p->tokens) return fail(KVQ_ERR_ARG, "tokens must be a device pointer");
  if (p->mask) {
    if (p->mask_rows < 1) return fail(KVQ_ERR_ARG, "mask_rows must be >= 1 (got %d)", p->mask_rows);
    if (p->mask_stride < (p->vocab + 31) / 32)
      return fail(KVQ_ERR_ARG, "mask_stride %lld smaller than %d words", (long long)p->mask_stride, (p->vocab + 31) / 32);
  }
  for (const void* x : {(const void*)p->tokens, (const void*)p->length, (const void*)p->prompt, (const void*)p->repetition,
                        (const void*)p->presence, (const void*)p->frequency, (const void*)p->bias_token,
                        (const void*)p->bias, (const void*)p->mask, (const void*)p->mask_row})
    if (reinterpret_cast<uintptr_t>(x) % 4 != 0) return fail(KVQ_ERR_ARG, "arrays must be 4-byte aligned");
  kvq::AdjustArgs a{};
  a.logits = p->logits;
  a.out = out;
  a.row_stride = p->row_stride;
  a.out_stride = out_row_stride;
  a.tokens = p->history > 0 ? p->tokens : nullptr;
  a.length = p->length;
  a.prompt = p->prompt;
  a.repetition = p->repetition;
  a.presence = p->presence;
  a.frequency = p->frequency;
  a.bias_token = p->bias_token;
  a.bias = p->bias;
  a.mask = p->mask;
  a.mask_row = p->mask_row;
  a.mask_stride = p->mask_stride;
  a.batch = p->batch; a.vocab = p->vocab; a.history = p->history; a.biases = p->biases; a.mask_rows = p->mask_rows;
  a.wide = p->history > kvq::kAdjustCount;
  // Every chunk of a row reads the row's whole history: long chunks where that is much, as
  // long as there are enough of them for every CU (512 rows of 128256 fp16, short and long
  // chunks: histories of 1024 tokens 62 us and 62, 4096 72 and 70, 8192 89 and 77).
  const int many = (p->vocab + 7 + kvq::kAdjustLong - 1) / kvq::kAdjustLong;
  a.chunk = !a.wide && p->history >= 4096 && (int64_t)p->batch * many >= 512 ? kvq::kAdjustLong : kvq::kAdjustChunk;
  a.nchunk = (p->vocab + 7 + a.chunk - 1) / a.chunk;
  // every row lies as far from a 16-byte border in as out
  const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(p->logits));
  a.runs = apart % (8 * size) == 0 && ((out_row_stride - p->row_stride) % 8 == 0 || p->batch == 1);
  const int e = kvq::launch_adjust(a, p->type, stream);
  return e ? kvq::hip_fail(e, "adjusted logits launch") : kvq::ok();
}
