/*
 * hps_mx4.h -- operators on frozen rows: rows held in microscaled 4-bit floating point, scored
 *              against queries of the same form, with log probabilities over the scores and
 *              their gradient.  Conventions as in hps.h: device pointers belong to the caller,
 *              nothing is allocated, calls enqueue work on `stream` and return, the GPU that
 *              holds the buffers is the current one.  Apart from hps_mx4_get these calls touch
 *              no table; any number of them may run at once, on any streams, as long as their
 *              outputs and workspaces are different buffers.  No output may overlap an
 *              input.  All of them may be captured into a HIP graph and replayed.
 *
 * What it is for: a trainer's rows (a catalogue of items or ads) are frozen for serving, in 17 bytes
 * for 32 values; pooled rows become queries; a request asks for the best rows of
 * the catalogue, a trainer for the log probability of the rows that were chosen, and for the
 * gradient that goes on into hps_push.  (A teacher's best rows as the given ones and minus its
 * probabilities as d_dlogp: distillation from the teacher's top scores.)
 *
 * The form: a row's values lie in blocks of 32, the last one of a row possibly shorter.  A block
 * has one scale, an 8-bit exponent byte b that stands for 2^(b - 127), and a 4-bit code per
 * value: sign, two exponent bits and one fraction bit, for the magnitudes 0, 0.5, 1, 1.5, 2, 3,
 * 4, 6.  The scale byte 255 marks a block that stands for NaN throughout.
 *   codes   [n, hps_mx4_row_bytes(dim)] bytes, two codes a byte, the earlier value in the low half;
 *           codes behind a row's last value are zero.  Aligned to 16 bytes (dim 12 and 16: 8, dim 4 and 8: 4)
 *   scales  [n, hps_mx4_row_scales(dim)] bytes, no alignment
 * dim as for a table: a multiple of 4, at most 1024.
 */
#ifndef HPS_MX4_H_
#define HPS_MX4_H_

#include "hps.h"

#ifdef __cplusplus
extern "C" {
#endif

/* What `type` says below (an int32_t there, as others than these two may be passed, and are refused). */
typedef enum { HPS_VALUES_F32 = 0, HPS_VALUES_BF16 = 1 } hps_value_type;

typedef struct {
  const uint8_t* d_codes;
  const uint8_t* d_scales;
  uint64_t n;               /* rows */
} hps_mx4_rows;

/* Bytes of codes and of scales a row takes; 0 for a dim that is not allowed. */
size_t hps_mx4_row_bytes(uint32_t dim);
size_t hps_mx4_row_scales(uint32_t dim);

/* Brings n rows of dim values into the 4-bit form.
 *   d_values   row i starts `stride` values after row i - 1; stride a multiple of 4, >= dim;
 *              float32 (16-byte aligned) or bfloat16 (8-byte aligned) by `type`
 *   d_rounded  [n, dim] float32 (16-byte aligned) or NULL: the values the codes stand for
 * A block's scale is the power of two of its largest magnitude, divided by 4 (never below
 * 2^-127); values are rounded to the nearest code, ties to the even one, and what lies above 6
 * scales becomes 6.  A block with an infinite value or a NaN gets the scale byte 255.
 * Errors: HPS_EINVAL. */
hps_status hps_mx4_quantize(const void* d_values, int32_t type, uint64_t n, uint32_t dim, uint64_t stride,
                            uint8_t* d_codes, uint8_t* d_scales, float* d_rounded, void* stream);

/* The values that n rows stand for: d_out [n, dim] float32, 16-byte aligned.  Errors: HPS_EINVAL. */
hps_status hps_mx4_dequantize(const hps_mx4_rows* rows, uint32_t dim, float* d_out, void* stream);

/* hps_get into the 4-bit form: the rows of d_keys [n] as codes and scales (of the table's dim)
 * without a float32 copy in between; nothing is created.  d_found_out [n] uint8; the rows of
 * absent keys (of all keys while the sticky device status is set) are zeros.  To be ordered
 * against the table's other calls as hps_get is.  Errors: HPS_EINVAL. */
hps_status hps_mx4_get(hps_table* t, const uint64_t* d_keys, uint64_t n, uint8_t* d_codes, uint8_t* d_scales,
                       uint8_t* d_found_out, void* stream);

/* What a query and a row of the catalogue give:
 *   score = scale * <query, row> + bias[row],  rounded to float32 once (the product of the
 * held values is summed in float32).  scale: a host value, at most 2^100 in magnitude; scores, and the
 * products before they are scaled, should stay below 2^126 (beyond, results may be NaN).
 *   d_bias [rows] float32 or NULL.  A bias that is not finite takes its row out: its score is
 *   -infinity, whatever its codes and the query's are.  The lowest finite value is a bias like any other.
 * At most 2^20 queries and fewer than 2^31 rows; either may be 0. */

/* All scores: d_out [queries, rows], row i `stride` values after row i - 1 (stride >= rows), float32
 * (4-byte aligned) or bfloat16 (2-byte aligned, each score rounded to the nearest) by `type`.
 * Errors: HPS_EINVAL. */
hps_status hps_mx4_scores(const hps_mx4_rows* queries, const hps_mx4_rows* rows, uint32_t dim, float scale,
                          const float* d_bias, void* d_out, int32_t type, uint64_t stride, void* stream);

/* Over the scores of each query, none of which is stored:
 *   d_lse     [queries] float32: log of the sum of exp(score)
 *   d_entropy [queries] float32: entropy of the distribution exp(score - lse)
 *   d_given   [queries, n_given] int32 row numbers or NULL (n_given 0), d_logp [queries, n_given]
 *             float32: score - lse of the given rows.  A negative number is padding and gets 0; a number
 *             beyond the last row gets NaN
 *   top       number of best rows wanted, at most HPS_MX4_MAX_TOP; d_top_index [queries, top] int32,
 *             d_top_logp [queries, top] float32 (both may be NULL for top = 0): row numbers and
 *             score - lse of the rows with the highest scores, best first, the lower number first
 *             among equal scores.  Where fewer rows are left: -1 and -infinity
 * A query that no row is left for: lse -infinity, entropy 0, logp -infinity.  A query that meets a
 * NaN score: lse, entropy, logp (but -infinity of a row that is taken out, and 0 of padding) and top_logp are NaN, and
 * the best rows are those among the others.
 *   d_workspace  hps_mx4_logprobs_bytes() bytes (0 for arguments that are not allowed), 256-byte aligned; its
 *                contents do not matter before and after.
 * Two calls with the same inputs give the same bits.  Errors: HPS_EINVAL, HPS_ENOMEM. */
#define HPS_MX4_MAX_TOP 64u
size_t hps_mx4_logprobs_bytes(uint64_t n_queries, uint64_t n_rows, uint32_t dim, uint32_t top);
hps_status hps_mx4_logprobs(const hps_mx4_rows* queries, const hps_mx4_rows* rows, uint32_t dim, float scale,
                            const float* d_bias, const int32_t* d_given, uint32_t n_given, uint32_t top,
                            float* d_lse, float* d_entropy, float* d_logp, int32_t* d_top_index, float* d_top_logp,
                            void* d_workspace, size_t workspace_bytes, void* stream);

/* The gradient of sum(d_dlogp * logp) + sum(d_dentropy * entropy) with respect to the values that the
 * queries' codes stand for: d_dqueries [queries, dim] float32, 16-byte aligned.
 *   d_lse, d_entropy  what hps_mx4_logprobs gave for the same arguments (d_entropy may be NULL if
 *                     d_dentropy is; with it the probabilities are a little more exact)
 *   d_given, d_dlogp  [queries, n_given] (both NULL: n_given 0); a row given twice counts twice; where d_given is no
 *                     row's number, or one of a row that is taken out, d_dlogp is not used
 *   d_dentropy        [queries] or NULL
 * A query that no row is left for has a gradient of 0, one that meets a NaN score of NaN.
 *   d_workspace       hps_mx4_logprobs_backward_bytes() bytes, 256-byte aligned
 * Two calls with the same inputs give the same bits; those of a query may depend on which others share the call (by less than
 * 2^-16 of the rows' magnitudes, weighted as they count).  Errors: HPS_EINVAL, HPS_ENOMEM. */
size_t hps_mx4_logprobs_backward_bytes(uint64_t n_queries, uint64_t n_rows, uint32_t dim);
hps_status hps_mx4_logprobs_backward(const hps_mx4_rows* queries, const hps_mx4_rows* rows, uint32_t dim, float scale,
                                     const float* d_bias, const float* d_lse, const float* d_entropy,
                                     const int32_t* d_given, const float* d_dlogp, uint32_t n_given,
                                     const float* d_dentropy, float* d_dqueries, void* d_workspace,
                                     size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HPS_MX4_H_ */
