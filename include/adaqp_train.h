/*
 * adaqp_train.h - what a network that classifies nodes has besides the layers of adaqp.h and adaqp_dense.h (AdaQP, arXiv 2306.01381, trains such networks:
 * Sec. 5 "Settings"): rows of a table at its beginning, dropout between its layers, products in more than 4 bits, log probabilities of classes at its end.
 *
 *   embedding         rows of a table by their ids, and the table's gradient by ids that were sorted on the GPU
 *   dropout           by a counter-based generator; nothing is stored, the backward pass is the same call
 *   matrices in 8 bits   e4m3 codes that share a power of two over 128 columns: written from rows, from columns or from both in one pass, read back,
 *                     multiplied on the matrix cores
 *   log probabilities of given classes, with entropy, the likeliest classes, and the logits' gradient
 *
 * Conventions are those of adaqp_dense.h: device pointers, buffers and workspaces of the caller, work only enqueued, errors found on the host before
 * anything is launched, counts of zero are no-ops.  Matrices of F32 or BF16 elements are row-major with a pitch ld >= columns, counted in
 * elements; rows of an output that is line-padded are written in whole lines, zeros behind the last column, of any other output only its columns are.
 * Reads stay between a matrix's first and last element.  Sums and statistics are held in 32 bits or more and rounded once, to nearest, when they are stored.
 * Results depend on shapes, layouts and values alone: repeated calls give the same bits.
 */
#ifndef ADAQP_TRAIN_H
#define ADAQP_TRAIN_H

#include "adaqp_dense.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------------------------------------- */
/* Embedding.                                                                                              */
/* ---------------------------------------------------------------------------------------------------- */

/* out_i = scale * table_{ids[i]}, rounded to `type`; zeros where ids[i] is outside [0, n_entries): a place without an entry.
 *   table_dev   [n_entries, ldt] of table_type;  ids_dev [n_ids] int32;  out_dev [n_ids, ldo] of type, not overlapping the table
 * Errors: EINVAL (also: scale not finite), ESIZE (2^31 ids or entries, more than 2^30 columns), EHIP. */
int adaqp_embedding_forward(const void *table_dev, int64_t ldt, int64_t n_entries, int32_t dim, int32_t table_type, const int32_t *ids_dev, int64_t n_ids,
                            float scale, void *out_dev, int64_t ldo, int32_t type, void *stream);

/* Bytes of workspace adaqp_embedding_sort needs (a multiple of 256).  Errors: EINVAL, ESIZE. */
int adaqp_embedding_sort_workspace_bytes(int64_t n_ids, int64_t n_entries, int64_t *bytes_out);

/* The places of n_ids ids in ascending order of their ids, equal ids in ascending order of places: sorted_dev[k] = ids[order_dev[k]].  Ids outside [0, n_entries) come
 * last, as n_entries.  Both written, [n_ids] int32; neither may overlap ids.
 * Errors: EINVAL, ESIZE (workspace too small, 2^31 ids or entries), EHIP. */
int adaqp_embedding_sort(const int32_t *ids_dev, int64_t n_ids, int64_t n_entries, int32_t *sorted_dev, int32_t *order_dev,
                         void *workspace_dev, int64_t workspace_bytes, void *stream);

/* Bytes of workspace adaqp_embedding_backward needs (a multiple of 256).  Errors: EINVAL, ESIZE. */
int adaqp_embedding_backward_workspace_bytes(int64_t n_ids, int32_t dim, int64_t *bytes_out);

/* dtable_e = scale * (the sum of dy_i over all i with id e), for all n_entries entries (zeros where there is no such i), or with `accumulate` added to what is there
 * (entries without i, and the padding of rows, are not touched).
 *   dy_dev                 [n_ids, lddy] of type
 *   sorted_dev, order_dev  as adaqp_embedding_sort wrote them for n_entries.  A place outside [0, n_ids) adds nothing, an id outside [0, n_entries) neither.
 *   dtable_dev             [n_entries, ldd] fp32
 * Sums are taken in ascending order of places, in fixed parts.
 * Errors: EINVAL (also: scale not finite), ESIZE (workspace too small, 2^31 ids or entries, more than 2^30 columns), EHIP. */
int adaqp_embedding_backward(const void *dy_dev, int64_t lddy, int64_t n_ids, int32_t dim, int32_t type, const int32_t *sorted_dev, const int32_t *order_dev,
                             int64_t n_entries, float scale, int32_t accumulate, float *dtable_dev, int64_t ldd,
                             void *workspace_dev, int64_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------------- */
/* Dropout.                                                                                                */
/* ---------------------------------------------------------------------------------------------------- */

/* y_ij = add_ij + (r_ij >= t ? x_ij * (2^16 / (2^16 - t)) : 0),  t = p * 2^16 to the nearest integer (halves up): an element is dropped with the probability t / 2^16, and
 * the expected value of what is added is x itself.  With t = 2^16 all are dropped.  A dropped infinity or NaN leaves nothing.
 * r_ij = r16(seed + *counter, first_row + i, j), Philox4x32-10 as in adaqp_quantize_pack with the last counter word 0x44524f50 and the row's upper half in the third.
 * The gradient of x is the same call on y's gradient, without `add`.
 *   add_dev       [n_rows, lda] of type; NULL: zeros
 *   first_row     the number of x's first row: rows that are dropped in several calls get the numbers of one
 *   counter_dev   NULL or a number in device memory that is added to the seed when the call runs: a captured call draws other numbers when it is changed between replays
 *   y_dev         may be x or add (same pitch)
 * Errors: EINVAL (also: p outside [0, 1]), ESIZE (more than 2^30 columns), EHIP. */
int adaqp_dropout(const void *x_dev, int64_t ldx, const void *add_dev, int64_t lda, int64_t n_rows, int32_t dim, int32_t type, double p, uint64_t seed,
                  int64_t first_row, const uint64_t *counter_dev, void *y_dev, int64_t ldy, void *stream);

/* ---------------------------------------------------------------------------------------------------- */
/* Matrices in 8 bits.                                                                                     */
/* ---------------------------------------------------------------------------------------------------- */

/* An 8-bit matrix of n_rows rows and n_cols columns is two arrays.
 *   codes   [n_rows][128 * ceil(n_cols / 128)] bytes in e4m3 (sign, 4 bits of exponent with bias 7, 3 of fraction; the largest is 448, 0x7F and 0xFF are NaN).
 *           Columns from n_cols on have code 0.
 *   scales  [ceil(n_cols / 128)][16 * ceil(n_rows / 16)] bytes: of row r and the 128 columns 128 b .. 128 b + 127 the byte at [b][r] = e + 127: the values are those of
 *           the codes times 2^e.  255: the block is NaN.  Rows from n_rows on have byte 0.
 * Both begin at a multiple of 16 bytes. */
#define ADAQP_F8_BLOCK 128
int64_t adaqp_f8_code_bytes(int64_t n_rows, int64_t n_cols);       /* of the two arrays; -1 for negative counts and beyond 2^31 - 1 */
int64_t adaqp_f8_scale_bytes(int64_t n_rows, int64_t n_cols);

#define ADAQP_F8_ROWS 0
#define ADAQP_F8_TILES 1

/* Writes a matrix (x_dev [n_rows, ld] of `type`) as an 8-bit matrix and / or its transpose as one, in one pass over x.
 * A block is 128 columns of a row (ROWS; for the transpose 128 rows of a column), or 128 columns of 128 rows (TILES: the transpose holds the same values).  Per block,
 * m = the largest magnitude: e = the smallest, at least -127, with m <= 448 * 2^e, and each value / 2^e to the nearest code, ties to the even one.  Nothing is clipped, and a power of
 * two costs the codes, which are floating-point numbers, none of their bits.  With e = 120 (m beyond 1.75 * 2^127) 240 stands in the place of 256: 2^128 is no fp32 number.  A block with an infinity or NaN: scale byte 255, codes 0.
 *   codes_dev, scales_dev       the matrix; both NULL: not wanted
 *   codes_t_dev, scales_t_dev   its transpose (n_cols rows, n_rows columns); both NULL: not wanted
 * Errors: EINVAL, ESIZE (2^31 rows or columns and more), EHIP. */
int adaqp_f8_quantize(const void *x_dev, int64_t ld, int64_t n_rows, int64_t n_cols, int32_t type, int32_t blocks,
                      uint8_t *codes_dev, uint8_t *scales_dev, uint8_t *codes_t_dev, uint8_t *scales_t_dev, void *stream);

/* The values of an 8-bit matrix: x_dev [n_rows, ld] of `type`, written.  fp32 holds all of them exactly, but for those from 2^128 on, which adaqp_f8_quantize writes none of and
 * which are infinite.  Errors: EINVAL, ESIZE, EHIP. */
int adaqp_f8_dequantize(const uint8_t *codes_dev, const uint8_t *scales_dev, int64_t n_rows, int64_t n_cols,
                        void *x_dev, int64_t ld, int32_t type, void *stream);

/* Bytes of workspace adaqp_f8_matmul needs (a multiple of 256; 0 where the product is not split over k).  Errors: EINVAL, ESIZE. */
int adaqp_f8_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t *bytes_out);

/* out[i, j] = sum_k a[i, k] * b[j, k]: both operands 8-bit matrices of k columns, a of m rows, b of n rows; out_dev [m, ldo] of `type`.
 * Sums are fp32: one that passes fp32's range on its way is infinite.  With BF16 outputs of more than 32 rows the products of eight columns 8 i .. 8 i + 7 are first added
 * to 14 bits of the largest of them (each loses less than 2^-13 of that), as the matrix cores do with such codes; with F32 outputs and with few rows products and sums are fp32's, and values
 * below 2^-126 may count as zeros.  So a row of a BF16 output may have other last bits in a matrix of more than 32 rows than in one of fewer.  With k = 0 the sum is empty and out is zeros.  A NaN block gives NaN in its row (of a) or column (of b).
 * Where few output tiles would leave the GPU idle, k is cut and the parts, held in the workspace in fp32, are added in order.
 * Errors: EINVAL, ESIZE (workspace too small; 2^31 rows and more; more than 2^24 columns), EHIP. */
int adaqp_f8_matmul(const uint8_t *a_codes_dev, const uint8_t *a_scales_dev, int64_t m,
                    const uint8_t *b_codes_dev, const uint8_t *b_scales_dev, int64_t n, int64_t k,
                    void *out_dev, int64_t ldo, int32_t type, void *workspace_dev, int64_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------------- */
/* Log probabilities.                                                                                      */
/* ---------------------------------------------------------------------------------------------------- */

#define ADAQP_LOGPROB_MOST_TOP 32

/* Bytes of workspace adaqp_logprob_forward needs (a multiple of 256; 0 where no row is split).  Errors: EINVAL, ESIZE. */
int adaqp_logprob_workspace_bytes(int64_t n_rows, int32_t n_classes, int32_t n_top, int64_t *bytes_out);

/* For each row x of n_classes logits:  max = the largest x_j,  others = the sum of exp(x_j - max) over all j but one with x_j = max,  rest = log(1 + others),
 *     logp_j = (x_j - max) - rest,   entropy = rest - sum_j (x_j - max) exp(x_j - max) / (1 + others) = - sum_j exp(logp_j) logp_j.
 * Without the one, what is far below 1 keeps its digits: the log probability of a class that is all but certain, too.
 *   logits_dev    [n_rows, ld] of type; -inf: a class that is ruled out, of probability 0
 *   targets_dev   [n_rows] int32; outside [0, n_classes): no class is given.  NULL: none is
 *   logp_dev      [n_rows] fp32: logp of the target, 0 without one; NULL: not wanted
 *   entropy_dev   [n_rows] fp32; NULL: not wanted
 *   stats_dev     [n_rows][2] fp32 = { max, rest }; NULL: not wanted
 *   n_top         how many of the largest logits are wanted, with their classes, in descending order, equal ones in ascending order of classes (-0 and 0 are equal; NaN is above all):
 *                 top_logp_dev, top_class_dev [n_rows][n_top] fp32 and int32.  0: none, both NULL
 * A row that is -inf throughout: logp and top_logp -inf (0 without a target), entropy 0, stats { -inf, 0 }.  A row with NaN or +inf: logp (of a target that is given), entropy, top_logp and
 * rest are NaN.
 * Errors: EINVAL (also: n_top above n_classes or ADAQP_LOGPROB_MOST_TOP), ESIZE (workspace too small, more than 2^30 classes), EHIP. */
int adaqp_logprob_forward(const void *logits_dev, int64_t ld, int64_t n_rows, int32_t n_classes, int32_t type, const int32_t *targets_dev,
                          float *logp_dev, float *entropy_dev, float *stats_dev, int32_t n_top, float *top_logp_dev, int32_t *top_class_dev,
                          void *workspace_dev, int64_t workspace_bytes, void *stream);

/* With p_j = exp(logp_j):  dlogits_j = scale * (dlogp * ([j is the target] - p_j) - dentropy * p_j * (logp_j + entropy)); the first term only in rows with a target.
 *   stats_dev, entropy_dev   as adaqp_logprob_forward wrote them; entropy_dev may be NULL where dentropy_dev is
 *   dlogp_dev                [n_rows] fp32; NULL: ones
 *   dentropy_dev             [n_rows] fp32; NULL: zeros
 *   dlogits_dev              [n_rows, ldd] of type; may be logits (same pitch)
 * Rows without a target and dentropy_dev, and rows that are -inf throughout: zeros.  Other rows with NaN or +inf: NaN.  A loss that is the mean of n rows' -logp takes scale = -1 / n.
 * Errors: EINVAL (also: scale not finite), ESIZE (more than 2^30 classes), EHIP. */
int adaqp_logprob_backward(const void *logits_dev, int64_t ld, int64_t n_rows, int32_t n_classes, int32_t type, const int32_t *targets_dev,
                           const float *stats_dev, const float *entropy_dev, const float *dlogp_dev, const float *dentropy_dev, float scale,
                           void *dlogits_dev, int64_t ldd, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ADAQP_TRAIN_H */
