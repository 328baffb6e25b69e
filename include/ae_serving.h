/*
 * ae_serving.h -- C ABI of the operators around attention with a key/value
 * cache, for AMD MI355X (gfx950): rotary positions, a paged cache that is
 * quantised as it is written, attention of a batch's newest tokens over that
 * cache, and the same behind a prefix that the whole batch shares.
 *
 * Conventions are those of ae_attn.h: entry points are host functions that
 * return a status, never throw and never abort; handles are host memory and
 * immutable (calls on one handle may run concurrently); pointers marked
 * "device" are device memory owned by the caller; work is enqueued on `stream`
 * and the call returns without waiting; nothing is allocated on the device.
 * ae_attn_last_error() has the message of the last failure.  The launch goes to
 * the current device, which has to be the one of the pointers and the stream.
 */
#ifndef AE_SERVING_H
#define AE_SERVING_H

#include "ae_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Strides {0, 0, 0} mean contiguous, here as in ae_attn.h.  {AE_ONE_ROW, 0, 0} says that they really are 0: every row of the
 * tensor is the one at its pointer (a vector expanded over batch, heads and rows).  For tensors that are read; an output is
 * refused with it. */
#define AE_ONE_ROW INT64_MIN

/* ---- Rotary positions -----------------------------------------------------
 * Every pair (x1, x2) of a row's first rot_dim elements is turned by the angle
 * of its frequency at the row's position p, and stretched:
 *     y1 = amplitude * (x1 cos(p f_i) - x2 sin(p f_i))
 *     y2 = amplitude * (x2 cos(p f_i) + x1 sin(p f_i))      i = 0 .. rot_dim/2 - 1
 * AE_ROTARY_HALF pairs element i with element i + rot_dim/2, AE_ROTARY_INTERLEAVED
 * element 2i with element 2i + 1.  Elements from rot_dim on are copied.  The
 * backward pass turns back (the transposed map): dx1 = amplitude * (dy1 cos + dy2
 * sin), dx2 = amplitude * (dy2 cos - dy1 sin).
 * Frequencies are the caller's (host, doubles): scaling for long contexts is a
 * choice of frequencies and amplitude.  Angles are exact for every 32-bit position:
 * p f / 2 pi is formed modulo 1 in 64-bit integers; sine and cosine are good to 1e-7, products
 * are formed in 32 bits and rounded once.
 *
 *   Q, K       device, [B, H_q, L, D] and [B, H_k, L, D], both of desc.dtype;
 *              K and K_out are NULL exactly when H_k is 0;
 *   positions  device, int32, position of row l of batch entry b at
 *              [b * position_stride + l] (stride 0: shared by the batch);
 *   outputs    same shapes and type; an output may be its own input (same
 *              pointer and strides), and must not overlap anything else.
 * Strides are in elements, {batch, head, row}, all 0 meaning contiguous, AE_ONE_ROW
 * and two 0 one row for all; the last dimension is contiguous.  Any alignment of at least the element's own is
 * taken; 16-byte aligned rows and pieces (pointers, strides, rot_dim / 2 and D -
 * rot_dim whole multiples of 16 bytes) run the wide kernel.                  */
typedef struct ae_rotary ae_rotary_t;
typedef enum { AE_ROTARY_HALF = 0, AE_ROTARY_INTERLEAVED = 1 } ae_rotary_layout_t;
typedef enum { AE_ROWS_BF16 = 0, AE_ROWS_F32 = 1 } ae_rows_dtype_t;
#define AE_MAX_ROT_DIM 256

typedef struct {
  int32_t B, H_q, H_k, L; /* H_k >= 0 */
  int32_t D, rot_dim;     /* rot_dim even, 2 .. min(D, AE_MAX_ROT_DIM); D <= 1024 */
  ae_rotary_layout_t layout;
  ae_rows_dtype_t dtype;
  const double *frequencies; /* host, rot_dim / 2 values of magnitude <= 6 (radians a position), copied by create */
  double amplitude;          /* finite */
  int64_t q_stride[3], k_stride[3], q_out_stride[3], k_out_stride[3]; /* >= 0, or AE_ONE_ROW, 0, 0 */
  int64_t position_stride;   /* >= 0 */
} ae_rotary_desc_t;

ae_status_t ae_rotary_create(const ae_rotary_desc_t *desc, ae_rotary_t **out);
ae_status_t ae_rotary_forward(const ae_rotary_t *h, const void *Q, const void *K, const int32_t *positions,
                              void *Q_out, void *K_out, hipStream_t stream);
/* dQ_out and dK_out have the layout of Q_out and K_out, dQ and dK that of Q and K. */
ae_status_t ae_rotary_backward(const ae_rotary_t *h, const void *dQ_out, const void *dK_out, const int32_t *positions,
                               void *dQ, void *dK, hipStream_t stream);
ae_status_t ae_rotary_destroy(ae_rotary_t *h); /* NULL is allowed */

/* ---- Paged key/value cache ------------------------------------------------
 * The cache of one layer is four device buffers of the caller:
 *   K_pages  [n_pages, H_kv, page_size, D_qk], V_pages [n_pages, H_kv, page_size, D_v],
 *            contiguous, 16-byte aligned, of desc.dtype;
 *   K_exp, V_exp  [n_pages, H_kv, page_size] bytes, 4-byte aligned (8-bit caches; else NULL).
 * A slot is page * page_size + place.  Which page holds which tokens is the
 * caller's affair.
 *
 * AE_CACHE_BF16 keeps rows as they are.  AE_CACHE_E4M3 keeps a row x of a head as
 * e4m3 values q (finite up to 448) and a power of two 2^k: k is the smallest number
 * >= -126 for which the row's largest finite magnitude is at most 448 * 2^k, the byte is
 * k + 127, and q = x / 2^k rounded to nearest even -- the division is exact, so a
 * value is rounded once.  A NaN or infinite element becomes NaN.  Values read back,
 * q * 2^k, are exact in bfloat16 (down to its smallest numbers, where they round; up to
 * its largest, where a value of 248 * 2^120 or more is rounded up to 2^128 and reads back
 * as an infinity).
 *
 * ae_cache_append writes row (b, l) of every head of K and V, [B, H_kv, L, D]
 * bfloat16, to slot slots[b * slot_stride + l]; a slot outside [0, n_pages *
 * page_size) is skipped.  Slots of one call that are not skipped must differ: of
 * two equal ones it is not defined which row's values and which row's exponent stay.
 * ae_cache_read is the way back: rows of K and V from those slots, as bfloat16;
 * zeros for a slot outside the range.  Reading the same slot more than once is fine.
 * K, V: device, 16-byte aligned, strides {batch, head, row} in elements, each a multiple of 8
 * (all 0: contiguous; AE_ONE_ROW, 0, 0: one row, for append).  slots: device, int32.                                */
typedef struct ae_cache ae_cache_t;
typedef enum { AE_CACHE_BF16 = 0, AE_CACHE_E4M3 = 1 } ae_cache_dtype_t;
typedef struct {
  int32_t n_pages;   /* >= 1, n_pages * page_size < 2^31 */
  int32_t page_size; /* 16, 32, 64, 128 or 256 */
  int32_t H_kv, D_qk, D_v; /* head dims 64/64, 128/128 or 192/128 */
  ae_cache_dtype_t dtype;
} ae_cache_desc_t;

ae_status_t ae_cache_create(const ae_cache_desc_t *desc, ae_cache_t **out);
ae_status_t ae_cache_append(const ae_cache_t *h, const void *K, const int64_t k_stride[3], const void *V,
                            const int64_t v_stride[3], int32_t B, int32_t L, const int32_t *slots, int64_t slot_stride,
                            void *K_pages, void *V_pages, void *K_exp, void *V_exp, hipStream_t stream);
ae_status_t ae_cache_read(const ae_cache_t *h, const void *K_pages, const void *V_pages, const void *K_exp,
                          const void *V_exp, int32_t B, int32_t L, const int32_t *slots, int64_t slot_stride,
                          void *K, const int64_t k_stride[3], void *V, const int64_t v_stride[3], hipStream_t stream);
ae_status_t ae_cache_destroy(ae_cache_t *h); /* NULL is allowed */

/* ---- Attention of the newest tokens over the paged cache -----------------
 * Softmax attention O = softmax(scale * Q K^T) V of the newest n_new tokens of B
 * sequences over everything cached for them (the parallel pattern of ae_attn.h
 * with L_q = n_new, bottom-right causal, keys and values in pages).  The
 * sequence's own keys, the newest tokens' included (append them first), are the
 * first lengths[b] positions of its page list: position j lies on page table[b][j / page_size].
 * Token t of the newest ones sees the first lengths[b] - n_new + 1 + t
 * of them; one that sees none gives a zero row with statistic -inf.  Query
 * head h reads k/v head h / (H_q / H_kv).
 *
 * Shared prefix (prefix_length > 0): all sequences have the prefix_length keys of
 * the page list prefix_table in front of their own, visible to every row; table and lengths then
 * hold what comes behind the prefix.  The prefix is read once for the rows of
 * all sequences together instead of once for each; the result is that of the
 * concatenated key lists.
 *
 *   Q          device, bf16 [B, H_q, n_new, D_qk], 16-byte aligned, strides multiples of 8 (AE_ONE_ROW, 0, 0: one row);
 *   table      device, int32 [B, table_width]; lengths  device, int32 [B];
 *   prefix_table  device, int32, ceil(prefix_length / page_size) entries; NULL without a prefix;
 *   O          device, [B, H_q, n_new, D_v], fp32 or (desc.out_dtype) bf16, 16-byte aligned,
 *              strides multiples of 8; strides of 0: contiguous;
 *   stats      device, fp32 [B, H_q, n_new], ln sum exp of the scaled scores; NULL: not written;
 *   workspace  device, 256-byte aligned, ae_cached_workspace_bytes (0: may be NULL); owned by
 *              the caller.  ae_cached_init_workspace has to be enqueued once before the first
 *              call that uses it (it clears counters, which every call leaves clear), and again
 *              after anything else has written there, another handle's calls included.
 *              Calls sharing it must not overlap.
 * At most 2^24 query rows, 2^30 keys a list, and 10^11 bytes of partial results (AE_ERR_UNSUPPORTED beyond).
 * lengths are read on the device: one outside [0, max_length] counts as the nearer
 * bound.  A page number outside [0, n_pages) is not followed: its keys count as hidden.
 * What lies in the cache behind a sequence's end may be anything, NaN included.
 * A NaN or infinity in a query row reaches that row alone (NaN, but for a row whose every score is -infinity: it counts as one without
 * keys); one in a cached row reaches the rows that see it and no others.
 *
 * Precision: scores, their softmax, sums, accumulators and partial results are fp32.  A weight is rounded once to bfloat16 (at most
 * 2^-8 of it, unbiased; 8-bit caches: after its product with the value row's power of two) for the product with the values, while
 * the sum that divides the row is that of the unrounded weights: an output is within 2^-8 sum_j p_j |v_j| of the exact one, and a
 * bf16 output is rounded once more.  stats are not affected.
 *
 * What the library chooses for chunk = 0 was fitted on calls whose lists are about max_length long, and, behind a prefix, on own
 * lists of up to 1024 keys: behind a prefix it cuts these into one or three ranges, which is too few for lists of many thousand
 * keys.  For those, give chunk, or name the prefix's pages in every sequence's list.  Every row of queries walks the list to its
 * end, also past the last key it sees: a long piece of a prompt is better read back (ae_cache_read) and put through ae_attn_forward
 * (1 x 32/8 heads of 128 over 8192 keys: 512 new tokens 111 us, that way 149; 4096 new tokens 1084 and 330). */
typedef struct ae_cached ae_cached_t;
typedef struct {
  int32_t B, H_q, n_new;  /* H_q a multiple of the cache's H_kv */
  int32_t table_width;    /* pages in a row of the table */
  int32_t max_length;     /* 1 .. table_width * page_size: no sequence has more keys of its own */
  int32_t prefix_length;  /* 0: no shared prefix */
  int32_t chunk;          /* 0: the library chooses; else the keys that one workgroup walks, a positive multiple of 128 */
  float scale;            /* non-zero; scale * log2(e) finite */
  ae_out_dtype_t out_dtype;
  int64_t q_stride[3], o_stride[3]; /* {batch, head, token} */
} ae_cached_desc_t;

ae_status_t ae_cached_create(const ae_cache_t *cache, const ae_cached_desc_t *desc, ae_cached_t **out); /* copies what it needs of the cache's handle */
ae_status_t ae_cached_workspace_bytes(const ae_cached_t *h, size_t *bytes);
ae_status_t ae_cached_init_workspace(const ae_cached_t *h, void *workspace, size_t workspace_bytes, hipStream_t stream);
ae_status_t ae_cached_forward(const ae_cached_t *h, const void *Q, const void *K_pages, const void *V_pages, const void *K_exp,
                              const void *V_exp, const int32_t *table, const int32_t *lengths, const int32_t *prefix_table,
                              void *O, float *stats, void *workspace, size_t workspace_bytes, hipStream_t stream);
/* What create chose: wavefronts of a workgroup, keys of a range of the sequences' own lists and of the prefix (0: none),
 * launches of a call.  Any pointer may be NULL.                              */
ae_status_t ae_cached_query(const ae_cached_t *h, int32_t *waves, int32_t *own_chunk, int32_t *prefix_chunk, int32_t *launches);
ae_status_t ae_cached_destroy(ae_cached_t *h); /* NULL is allowed */

#ifdef __cplusplus
}
#endif
#endif /* AE_SERVING_H */
