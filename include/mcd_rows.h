/* libmcd: operators on the rows between a layer's products.
 *
 * A program that serves many utterances of a Sec. 1 / Fig. 1 model (arXiv 2609.37007) over the paged cache of
 * mcd_cache.h and the products of mcd_tc.h has from here
 *
 *   mcd_norm_rows      residual sum, RMSNorm and the rounding to the next product's type, 8 bits with a scale per
 *                      row among them
 *   mcd_sample_rows    a token of every row of logits: temperature, top-k, top-p and min-p, from given random numbers
 *
 * Conventions are those of mcd.h: a status is returned, nothing aborts across the ABI.  Every call is asynchronous
 * on `stream` (a cudaStream_t of the current device, or NULL for the default stream), allocates nothing, needs no
 * workspace and can be captured into a graph.
 */
#ifndef MCD_ROWS_H
#define MCD_ROWS_H

#include "mcd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of rows: MCD_WEIGHT_F32, MCD_WEIGHT_BF16 and 8-bit floating point with 4 bits of exponent and 3 of mantissa
 * (largest value 448, no infinities). */
enum { MCD_E4M3 = 3 };

/* For every row: r = x + residual, stored in `sum`; v = r / sqrt(mean r^2 + eps) * gain; y = v.  Each is rounded once
 * (v comes from the unrounded r), sums are fp32.  With y_dtype MCD_E4M3 the row has a scale,
 * s = max(max |v| / 448, 2^-126), and y = v / s to the nearest value: y * s stands for v.  A row that holds an infinity
 * or NaN has, with `norm`, no finite v, and in 8 bits no finite y * s; nor has, with `norm`, one whose sum of squares
 * is above fp32's range (squares below it are lost: with eps 0, values below 1e-19).  Other rows are not touched by it.
 * The gain is multiplied last: r * gain may leave fp32's range where v does not.
 *   x          dev [n_rows][x_stride], x_dtype MCD_WEIGHT_F32 or MCD_WEIGHT_BF16
 *   residual, sum   dev [n_rows][stride], res_dtype likewise.  residual NULL: r = x (res_dtype is sum's).  sum
 *              NULL: not stored
 *   norm       0: v = r * gain, eps is not looked at (8 bits: the quantiser of any rows, weights among them)
 *   gain       dev float [width], or NULL for ones
 *   eps        >= 0, finite
 *   y          dev [n_rows][y_stride], y_dtype MCD_WEIGHT_F32, MCD_WEIGHT_BF16 or MCD_E4M3
 *   y_scale    dev float [n_rows] with MCD_E4M3, else not looked at
 * Strides are in elements, at least width; rows and gain are 16-byte aligned, width at most 16,384
 * (MCD_ERR_UNSUPPORTED otherwise).  sum may be residual, and sum or y may be x or residual, of the same type and
 * stride; apart from that an output overlaps neither an input nor the other outputs (MCD_ERR_INVALID_ARG; rows of one stride
 * may lie beside each other, of two strides what lies between each other's rows counts as overlapping).  No rows: MCD_OK. */
mcd_status mcd_norm_rows(int32_t n_rows, int32_t width, const void* x, int64_t x_stride, int32_t x_dtype,
                         const void* residual, int64_t residual_stride, void* sum, int64_t sum_stride,
                         int32_t res_dtype, int32_t norm, const float* gain, float eps, void* y, int64_t y_stride,
                         int32_t y_dtype, float* y_scale, void* stream);

/* One id of every logits row, drawn from the distribution that the row's settings leave.  In whole numbers, so that
 * any two implementations agree: with z = logit / T and exp32 the exponential of mcd.h, an id has the weight
 * W = floor(2^31 exp32(z - z_max)).  Ids are ranked by logit (descending), then id (ascending); what is left are the ids
 * of W > 0
 *   - among the first top_k of the ranking,
 *   - in its shortest prefix whose weights sum to at least ceil(top_p * S) (double; S: the weights of those top_k; at
 *     least 1), and
 *   - with W >= ceil(min_p * 2^31): at least min_p times the largest probability.
 * With M the sum of their weights, the drawn id is the first in ascending order whose running sum exceeds
 * min(floor(u * M), M - 1) (double).  (mcd_topk_softmax has the same set and order for top_k alone; its weights have 24 bits.)
 *   logits       dev [n_rows][stride] (elements), dtype MCD_WEIGHT_F32 or MCD_WEIGHT_BF16; -inf hides an id
 *   temperature  dev float [n_rows], NULL: 1.  0: the first id of the ranking (also where z leaves fp32's range)
 *   top_k        dev int32 [n_rows], NULL: off; so is a value below 1 or from vocab on
 *   top_p        dev float [n_rows], NULL: off; so is a value from 1 on.  0 and below: the first id of the ranking
 *   min_p        dev float [n_rows], NULL: off; so is a value of 0 or below.  Above 1 it is 1
 *   u            dev double [n_rows], in [0, 1)
 *   ids          dev int32 [n_rows]
 *   probs        dev float [n_rows], optional: W / M of the drawn id
 *   kept         dev int32 [n_rows], optional: how many ids were left
 *   err          dev int32, zeroed by the caller: MCD_ERR_INVALID_ARG when a row has a NaN, +inf or nothing but -inf, or a
 *                setting that is NaN or out of its range; such a row has id -1, probability 0 and 0 ids left;
 *                MCD_ERR_TIMEOUT if a search gave up (a fault of the library: the row's result is not to be used)
 * Rows are 16-byte aligned, vocab is at most 262,144 (MCD_ERR_UNSUPPORTED otherwise).  Outputs and err overlap nothing
 * (MCD_ERR_INVALID_ARG).  No rows: MCD_OK. */
mcd_status mcd_sample_rows(int32_t n_rows, int32_t vocab, const void* logits, int64_t stride, int32_t dtype,
                           const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                           const double* u, int32_t* ids, float* probs, int32_t* kept, int32_t* err, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MCD_ROWS_H */
