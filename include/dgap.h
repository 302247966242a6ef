/*
 * dgap — the logit-side runtime step of DGAP on AMD Instinct MI355X
 * (gfx950), the token drawn from the logits it leaves (dgap_sample), and the
 * Kullback-Leibler loss against a teacher's top logits, one term of what its
 * corrector is trained with (dgap_distill).  Plain C ABI, in the same library as
 * kvq.h.
 *
 * DGAP restores the local top-K candidate distribution of a decoder that
 * keeps a low-bit KV cache (Methodology, "DGAP Overview", online restoration
 * framework).  At each decode step it computes runtime features phi from the
 * quantized logits z^ alone, scores them with a detector,
 * r = sigmoid(f_theta(phi)) ("Distribution-Risk Detector"), and, only when
 * r > tau, predicts updates Delta for the window S = TopK(z^, K_b) with a
 * corrector g_psi from candidate features and phi, merging them back:
 * z~_j = z^_j + Delta_j for j in S, z~_j = z^_j otherwise ("Selective Top-K
 * Distribution Corrector", sparse merge).  The paper uses MLPs for both
 * modules and tau = 0.60 (ablations).  It leaves the features, the MLP
 * shapes and K_b open; this library fixes:
 *   - TopK: the K largest logits, largest first, equal logits by lower
 *     vocabulary index;
 *   - phi (DGAP_FEATURES = 12), with v_1 >= ... >= v_K the window's logits,
 *     p = softmax(z^) over the vocabulary and P_k = p at v_k, natural logs:
 *       0 entropy H = -sum p log p,  1 H / log V,  2 log P_1,
 *       3 sum_k P_k,  4 sum_{k<=8} P_k,  5 sum p^2,  6 v_1 - v_2,
 *       7 v_2 - v_3,  8 (v_1 - v_K) / (K - 1),  9 min_{k<8} (v_k - v_{k+1}),
 *       10 population standard deviation of v_1..v_K,
 *       11 entropy of P_1..P_K renormalized to sum 1 (0 log 0 = 0);
 *   - xi_k (DGAP_CAND_INPUTS = 5) for candidate k = 1..K: v_k - v_1,
 *     v_k - log-sum-exp(z^), (k - 1) / (K - 1), v_{k-1} - v_k (0 for k = 1),
 *     v_k - v_{k+1} (0 for k = K);
 *   - f_theta(phi) = w2 . relu(W1^T phi + b1) + b2 and
 *     g_psi(xi_k, phi) = w2' . relu(W1'^T [xi_k, phi] + b1') + b2', one
 *     hidden layer each, g_psi shared by the K candidates.
 *
 * Conventions: device pointers are caller-owned HIP device buffers; the
 * library allocates nothing; `stream` is a hipStream_t as void*, calls are
 * asynchronous and stream-ordered.  A non-OK status other than KVQ_ERR_HIP
 * launches nothing and leaves every buffer unchanged; kvq_last_error()
 * describes the failure.
 */
#ifndef DGAP_H
#define DGAP_H

#include <stddef.h>
#include <stdint.h>

#include "kvq.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DGAP_FEATURES 12
#define DGAP_CAND_INPUTS 5
#define DGAP_MIN_K 8
#define DGAP_MAX_K 256
#define DGAP_MAX_HIDDEN 64

/* Shapes, threshold and weights (device pointers, fp32, row-major). */
typedef struct {
  int32_t vocab;        /* V, K <= V <= 2^24 */
  int32_t k;            /* K_b, DGAP_MIN_K .. DGAP_MAX_K */
  int32_t hidden_det;   /* detector hidden units, 1 .. DGAP_MAX_HIDDEN */
  int32_t hidden_corr;  /* corrector hidden units, 1 .. DGAP_MAX_HIDDEN */
  float tau;            /* risk threshold: correct when r > tau */
  float det_b2;         /* detector output bias */
  float corr_b2;        /* corrector output bias */
  int32_t pad;
  const float* det_w1;  /* [DGAP_FEATURES][hidden_det] */
  const float* det_b1;  /* [hidden_det] */
  const float* det_w2;  /* [hidden_det] */
  const float* corr_w1; /* [DGAP_CAND_INPUTS + DGAP_FEATURES][hidden_corr]: rows 0..4 take xi, 5..16 phi */
  const float* corr_b1; /* [hidden_corr] */
  const float* corr_w2; /* [hidden_corr] */
} dgap_params;

/* Workspace bytes dgap_restore needs for `batch` rows of `vocab` logits and
 * window k; 0 if the shape is not supported. */
size_t dgap_workspace_bytes(int32_t batch, int32_t vocab, int32_t k);

/* Floats per row of dgap_restore's optional info output:
 *   [0] r, [1] 1 if the row was corrected else 0, [2] log-sum-exp of the
 *   row, [3] 0, [4 .. 4+12) phi, [16 .. 16+k) the window's vocabulary
 *   indices in TopK order (int32 bit patterns), [16+k .. 16+2k) Delta in the
 *   same order (0 when the row was not corrected). */
size_t dgap_info_floats(int32_t k);

/* One DGAP step on `batch` rows of fp32 logits, in place: logits is a
 * device array [batch][vocab], finite values; only the K entries of a
 * corrected row's window change.  ws: device scratch of ws_bytes >=
 * dgap_workspace_bytes, 16-byte aligned, contents undefined on entry and
 * exit.  info: NULL or a device array [batch][dgap_info_floats(k)].
 * Errors: KVQ_ERR_ARG (null params, pointers or weights, shapes out of
 * range, small or misaligned workspace), KVQ_ERR_UNSUPPORTED (vocab above
 * 2^24, or more than 32768 window candidates: ceil(vocab / 2048) * k),
 * KVQ_ERR_HIP (launch failure).  Results are bitwise reproducible. */
kvq_status dgap_restore(const dgap_params* p, float* logits, int32_t batch, void* ws, size_t ws_bytes,
                        float* info, void* stream);

/* Element types of the rows of logits below. */
typedef enum { DGAP_F32 = 0, DGAP_F16 = 1, DGAP_BF16 = 2 } dgap_type;

/* Rows of logits and how a token is drawn from each (device pointers; the
 * settings are arrays of `batch` values, one per row). */
typedef struct {
  const void* logits;       /* [batch] rows of `vocab` logits of `type`, row_stride elements apart */
  int64_t row_stride;       /* >= vocab */
  int32_t type;             /* dgap_type */
  int32_t batch;            /* >= 1 */
  int32_t vocab;            /* 1 .. 2^24 */
  int32_t pad;
  const float* temperature; /* T >= 0, finite; NULL: 1 */
  const int32_t* top_k;     /* NULL, or k < 1 or k >= vocab in a row: off */
  const float* top_p;       /* NULL, or p >= 1 in a row: off */
  const float* min_p;       /* NULL, or m <= 0 in a row: off */
  const float* uniform;     /* a number u in [0, 1) per row */
} dgap_sampling;

/* Workspace bytes dgap_sample needs; 0 if the shape is not supported. */
size_t dgap_sample_workspace_bytes(int32_t batch, int32_t vocab);

/* The next token of every row: token selection from the (restored) logits,
 * what a decode step does after dgap_restore ("DGAP Overview", online
 * restoration framework: decoding proceeds from z~).  In the row's descending
 * order, equal logits by lower index, with weights e^((z - z_max) / T):
 *   top-k keeps the first k; of their mass, top-p keeps the shortest beginning
 *   that holds at least p of it (one element at least); min-p keeps those of
 *   weight >= m (the largest alone where m > 1).  The token is the first of
 *   the kept ones up to and with which their mass is more than u times all of
 *   it (u is clipped to [0, 1 - 2^-24]).
 * T = 0 gives the largest logit.  tokens: device int32 [batch]; logprobs: NULL
 * or device fp32 [batch], the log of the token's share of the kept mass (0
 * where T = 0).  A logit of -inf is never drawn (a masked token).  A row
 * without a finite logit, with a NaN or +inf among them, or with a setting
 * that is NaN (T: negative or infinite, too) gives token -1 and log-probability
 * NaN.  Weights are taken to 24 bits and added up exactly in units of 2^-45 of
 * the largest (2^-38 for the largest vocabularies): a sampled step differs
 * from the exact one where u is within about 1e-7 of a border.
 * ws: device scratch of ws_bytes >= dgap_sample_workspace_bytes, 16-byte
 * aligned, contents undefined on entry and exit; calls that may overlap take
 * one each.  Errors: KVQ_ERR_ARG (null pointers, shapes or type out of range,
 * misaligned logits or workspace), KVQ_ERR_CAPACITY (workspace too small),
 * KVQ_ERR_UNSUPPORTED (vocab above 2^24, 2^22 chunks of 8192 logits or more),
 * KVQ_ERR_HIP.  Results are bitwise reproducible. */
kvq_status dgap_sample(const dgap_sampling* p, int32_t* tokens, float* logprobs, void* ws, size_t ws_bytes,
                       void* stream);

/* Most teacher entries per row. */
#define DGAP_MAX_TEACHER 256

/* A student's logits and a teacher's top logits (device pointers). */
typedef struct {
  const void* logits;     /* [rows] rows of `vocab` logits of `type`, row_stride elements apart */
  int64_t row_stride;     /* >= vocab */
  int32_t type;           /* dgap_type */
  int32_t rows;           /* >= 1 */
  int32_t vocab;          /* 1 .. 2^24 */
  int32_t k;              /* teacher entries per row, 1 .. DGAP_MAX_TEACHER */
  const float* teacher;   /* [rows][k] the teacher's logits */
  const int32_t* index;   /* [rows][k] their vocabulary indices */
  float temperature;      /* T > 0, finite, and so 1 / T */
  int32_t pad;
} dgap_distillation;

/* Workspace bytes dgap_distill needs; 0 if the shape is not supported. */
size_t dgap_distill_workspace_bytes(int32_t rows, int32_t vocab);

/* The loss of every row against the teacher's top logits, and its gradient:
 * the Kullback-Leibler term at temperature T that DGAP's corrector is trained
 * with against the FP16 decoder ("Selective Top-K Distribution Corrector",
 * corrector loss: KL(q^fp || q~)), taken over the whole vocabulary on the
 * student's side, so that it also tunes a model that will decode from a
 * low-bit cache:
 *   q = softmax(t / T) over the row's entries, p = softmax(z / T),
 *   loss[r] = T^2 sum_k q_k (log q_k - log p_{i_k}),
 *   grad[r][j] = grad_loss[r] T (p_j - sum_k q_k [i_k = j]).
 * An index outside [0, vocab) or a teacher logit of -inf stands for no entry
 * (rows of fewer entries); entries of one index add up; a row without entries
 * has loss and gradient 0; an entry's teacher logit of NaN or +inf makes the loss
 * NaN, and the gradient at the row's entries.  Logits are finite or -inf (p = 0:
 * a loss of +inf where the teacher has an entry there), of a row with entries one
 * finite at least.
 * loss: device fp32 [rows].  lse: NULL or device fp32 [rows], log sum e^(z/T)
 * for dgap_distill_backward.  grad: NULL (the loss alone) or device rows of
 * the logits' type, grad_row_stride >= vocab elements apart; it may be the
 * logits' own memory (row strides equal), but overlap them in no other way.
 * grad_loss: NULL (1) or device fp32 [rows].  ws: device scratch of ws_bytes
 * >= dgap_distill_workspace_bytes, 16-byte aligned, contents undefined on entry
 * and exit; calls that may overlap take one each.  Sums and logarithms are
 * fp32 or wider, the gradient is rounded once; results are bitwise
 * reproducible.  Errors: KVQ_ERR_ARG (null pointers, shapes, type or
 * temperature out of range, misaligned logits, grad or workspace),
 * KVQ_ERR_CAPACITY (workspace too small), KVQ_ERR_UNSUPPORTED (vocab above 2^24,
 * 2^22 chunks of 8192 logits or more), KVQ_ERR_HIP. */
kvq_status dgap_distill(const dgap_distillation* p, float* loss, float* lse, void* grad, int64_t grad_row_stride,
                        const float* grad_loss, void* ws, size_t ws_bytes, void* stream);

/* The gradient alone, from the lse of an earlier dgap_distill on the same
 * logits (a backward pass whose grad_loss was not known then).  Arguments,
 * results and errors as there; p is as exact as the fp32 lse is (2^-24 |lse|
 * relative), so a row's largest logit has to be a score, not a mask's lowest
 * value. */
kvq_status dgap_distill_backward(const dgap_distillation* p, const float* lse, const float* grad_loss, void* grad,
                                 int64_t grad_row_stride, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* DGAP_H */
