/*
 * ae_span.h -- C ABI of softmax attention over spans of keys, with capped and
 * distance-biased scores, forward and backward, for AMD MI355X (gfx950).
 *
 * Every query row sees one span of keys, [begin, end): documents packed behind
 * each other in a row, prefixes that are seen both ways, windows and the causal mask are such
 * spans.  For query row i of batch entry b and head h, with off = L_k - L_q,
 *     s_j  = scale q_i . k_j
 *     s'_j = cap tanh(s_j / cap)  (where there is a cap)  - slope_h |i + off - j|  (where there are slopes)
 *     O_i  = sum_j softmax_j(s') v_j      stats_i = ln sum_j exp(s'_j)      begin <= j < end
 * A row whose span is empty gives a zero row, the statistic -inf, and zero gradients.
 *
 * Conventions are those of ae_attn.h: entry points are host functions that
 * return a status, never throw and never abort; handles are host memory and
 * immutable (calls on one handle may run concurrently); pointers marked
 * "device" are device memory owned by the caller; work is enqueued on `stream`
 * and the call returns without waiting; nothing is allocated on the device, and calls
 * can be captured into a graph.  ae_attn_last_error() has the message of the last
 * failure.  The launch goes to the current device, which has to be the one of the
 * pointers and the stream.
 */
#ifndef AE_SPAN_H
#define AE_SPAN_H

#include "ae_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The span of query row i, cut to [0, L_k). */
typedef enum {
  AE_SPAN_ALL = 0,    /* every key                                            */
  AE_SPAN_CAUSAL = 1, /* j <= i + L_k - L_q                                   */
  AE_SPAN_WINDOW = 2, /* i + L_k - L_q - window < j <= i + L_k - L_q          */
  AE_SPAN_GIVEN = 3   /* key_begin[b, i] <= j < key_end[b, i], given per call  */
} ae_span_mask_t;

#define AE_MAX_SLOPE_HEADS AE_MAX_DECAY_HEADS
#define AE_MAX_SLOPE 128 /* (where the keys next to a key weigh 2^-184 of it) */

/*
 * Layouts (bf16 inputs, fp32 or bf16 output, last dimension contiguous):
 *   Q [B, H_q, L_q, D_qk]   K [B, H_kv, L_k, D_qk]   V [B, H_kv, L_k, D_v]   O [B, H_q, L_q, D_v]
 * Query head h reads k/v head h / (H_q / H_kv).  Strides are in elements,
 * {batch, head, row}, all 0 meaning contiguous; those of Q, K and V are multiples of 8,
 * those of O of 4, and a row stride is at least the head dim.  One (batch, head) slab
 * of Q, K or V spans less than 4 GiB.
 */
typedef struct {
  int32_t B, H_q, H_kv, L_q, L_k; /* >= 1; H_q a multiple of H_kv */
  int32_t D_qk, D_v;              /* 64/64, 128/128 or 192/128 */
  float scale;                    /* finite and non-zero */
  float cap;                      /* 0: none; else positive, with cap and scale / cap in the range of 32-bit numbers */
  const float *slopes;            /* host, [H_q] finite numbers below 10^30 times the scale, copied by create; NULL: none.  AE_ERR_UNSUPPORTED beyond AE_MAX_SLOPE in
                                   * magnitude, AE_MAX_SLOPE_HEADS heads or L_q + L_k = 2^24 */
  ae_span_mask_t mask;
  int32_t window;                 /* AE_SPAN_WINDOW: >= 1 */
  ae_out_dtype_t out_dtype;       /* of O */
  int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];
  int32_t kv_splits;              /* of ae_span_forward_split: ranges that a row's keys are cut into, 0 .. 256; 0: the library chooses */
} ae_span_desc_t;

typedef struct ae_span ae_span_t;

ae_status_t ae_span_create(const ae_span_desc_t *desc, ae_span_t **out);

/* One launch.  key_begin, key_end: device, int32, that of row i of batch entry b at
 * [b * span_stride + i] (0: shared by the batch); NULL unless the mask is
 * AE_SPAN_GIVEN.  Spans may come in any order and may overlap; sorted ones (neither beginnings nor ends ever fall)
 * cost least, as the tiles of keys between the first and the last one that 256 rows see are walked.
 * stats: device, fp32 [B, H_q, L_q] contiguous, or NULL.  Q, K, V, O: 16-byte aligned; outputs alias nothing.
 * Inputs are finite: a NaN or infinity in a row of V, as in ae_attn_forward, can reach rows that do not see it.
 *
 * Precision: scores, their modification, softmax, sums and accumulators are fp32; a weight is rounded once to bf16 for the
 * product with the values, while the sum that divides the row is that of the unrounded weights: an output is within 2^-8
 * sum_j p_j |v_j| of the exact one, and a bf16 output is rounded once more.  A capped score has a relative error of 3e-7 up to 0.6
 * of the cap (0.2, 0.1, 0.03 and 5e-4 of it where |scale| / cap is below 1.2e-4, 8e-6, 6e-8 and 7e-13) and an absolute one of 2e-7 of the cap beyond, or
 * everywhere where |scale| / cap is above 4e3 (caps up to 10^6; with larger ones sooner) and where |q . k| is above 10^18.  With
 * slopes the score of a key at distance x carries an error of up to 2^-21 |slope| (64 + x) besides, its weight as much of itself, and the statistic that of the keys
 * with most weight: an output is within (2^-8 + 2^-20 |slope| (64 + x)) sum_j p_j |v_j|.  For near keys that is next to nothing at usual slopes (3e-5 at 1) and 2^-8 at the
 * steepest; where rows see far keys alone, or the slope is negative, far keys count (measured at slope 1 and x = 65536: statistics are off by up to 8e-3, a quarter of that bound).
 * And a row's weights may be held at 2^-80 of their size with slopes: products with values below 2^-40 in magnitude can be lost then.          */
ae_status_t ae_span_forward(const ae_span_t *h, const void *Q, const void *K, const void *V, const int32_t *key_begin,
                            const int32_t *key_end, int64_t span_stride, void *O, float *stats, hipStream_t stream);

/* The same with the keys that 256 rows see cut into ranges, for calls of few workgroups (few rows and heads, many keys): each range's rows go to the workspace, and a
 * second launch combines them, in a fixed order.  workspace: device, 16-byte aligned, ae_span_workspace_bytes (0, where keys are not cut: may be
 * NULL, and the call is ae_span_forward), needs no initialisation.  Calls that share it must not overlap.               */
ae_status_t ae_span_workspace_bytes(const ae_span_t *h, size_t *bytes);
ae_status_t ae_span_forward_split(const ae_span_t *h, const void *Q, const void *K, const void *V, const int32_t *key_begin,
                                  const int32_t *key_end, int64_t span_stride, void *O, float *stats, void *workspace, size_t workspace_bytes,
                                  hipStream_t stream);

/* Gradients of sum(O * dO):
 *   P = exp(s' - stats), dV = P^T dO, dP = dO V^T, dS = P (dP - dO . O) (1 - tanh^2(s / cap)), dQ = scale dS K, dK = scale dS^T Q,
 * dK and dV summed over the query heads that share a k/v head; nothing is accumulated by atomics.  The slopes get no gradient.
 *   O, stats   as the forward pass wrote them;
 *   dO         device, bf16, 16-byte aligned, strides as for O's shape, multiples of 8 (all 0: contiguous);
 *   dQ, dK, dV device, contiguous, fp32 or bf16 (grad_dtype), 16-byte aligned, every element is written;
 *   workspace  device, 16-byte aligned, ae_span_backward_workspace_bytes, needs no initialisation.  Calls that share it must not overlap.
 * Two or three launches.  P and dS are rounded once to bf16 for the products.
 * With slopes P carries the relative error of the statistic that the forward pass wrote and of its own scores, each as above.
 * With O in bf16 its rounding enters dO . O: where a row sees few keys, dP - dO . O is a small difference of larger numbers, so
 * keep O in fp32 where such rows' gradients matter.                                                                    */
ae_status_t ae_span_backward_workspace_bytes(const ae_span_t *h, size_t *bytes);
ae_status_t ae_span_backward(const ae_span_t *h, const void *Q, const void *K, const void *V, const int32_t *key_begin,
                             const int32_t *key_end, int64_t span_stride, const void *O, const void *dO, const int64_t do_stride[3],
                             const float *stats, void *dQ, void *dK, void *dV, ae_out_dtype_t grad_dtype, void *workspace,
                             size_t workspace_bytes, hipStream_t stream);
ae_status_t ae_span_destroy(ae_span_t *h); /* NULL is allowed */

/* Spans of documents packed in rows of L tokens: document d of batch entry b is the tokens offsets[b][d] <= i < offsets[b][d + 1], d = 0 ..
 * n_docs - 1 (offsets never fall, a document may be empty; tokens outside all of them are padding and see nothing).
 *   mask ALL     a token sees its document;
 *   mask CAUSAL  its document up to itself;
 *   mask WINDOW  of that the nearest `window` keys.
 * prefix (may be NULL; ALL and CAUSAL): the first prefix[b][d] tokens of the document are seen by all of it.
 * offsets, prefix: device, int32, batch entries offset_stride and prefix_stride apart (0: shared); key_begin, key_end: device, int32 [B, L].
 * One launch.                                                                                                           */
ae_status_t ae_span_documents(int32_t B, int32_t L, int32_t n_docs, const int32_t *offsets, int64_t offset_stride, const int32_t *prefix,
                              int64_t prefix_stride, ae_span_mask_t mask, int32_t window, int32_t *key_begin, int32_t *key_end,
                              hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* AE_SPAN_H */
