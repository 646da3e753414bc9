/*
 * adaqp_dense.h - the dense half of a layer, next to the message path and aggregation of adaqp.h (AdaQP, arXiv 2306.01381, Sec. 2.1 Eq. 3's
 * outer part and Sec. 5 "Settings", whose models have a layer norm in every layer): what a training program does with the aggregated rows.
 *
 *   layer norm        forward and backward, with the gradients of its two parameter vectors
 *   matrices in 4 bits   MX blocks (32 values of 4 bits that share a power of two): written from rows, from columns or from both in one pass,
 *                     rounded to nearest or stochastically, read back, multiplied on the matrix cores
 *   orthogonalised update   Newton-Schulz steps on the gradient of a weight matrix
 *
 * Conventions are those of adaqp.h: device pointers, buffers and workspaces of the caller, work only enqueued, errors found on the host
 * before anything is launched, counts of zero are no-ops.  Matrices of F32 or BF16 elements are row-major with a pitch ld >= columns, counted in
 * elements.  Line-padded (base on a 128-byte line, pitch a multiple of 128 bytes) is the preferred layout: such a matrix owns all of its lines,
 * and of one that is written the rows are written in whole lines, zeros behind the last column.  Of any other output only its columns are
 * written.  Sums, statistics and products are held in 32 bits or more and rounded once, to nearest, when they are stored.
 * Results depend on shapes, layouts and values alone: repeated calls give the same bits.
 */
#ifndef ADAQP_DENSE_H
#define ADAQP_DENSE_H

#include "adaqp.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum adaqp_type {
    ADAQP_F32 = 0,
    ADAQP_BF16 = 1
} adaqp_type;

/* ---------------------------------------------------------------------------------------------------- */
/* Layer norm.                                                                                             */
/* ---------------------------------------------------------------------------------------------------- */

/* For each row:  mean = sum_j x_j / dim,  rstd = 1 / sqrt(sum_j (x_j - mean)^2 / dim + eps),
 *     y_j = (x_j - mean) * rstd * gamma_j + beta_j,   stats[row] = { mean, rstd }.
 *   x_dev, y_dev   [n_rows, ldx], [n_rows, ldy] of `type`; y may be x (same pitch)
 *   gamma_dev, beta_dev   [dim] fp32; NULL: ones, zeros
 *   stats_dev      [n_rows][2] fp32, written; NULL: not wanted
 * Infinities and NaN give NaN in their own row only.
 * Errors: EINVAL (also: eps negative or not finite, an unknown type, a pointer that is not aligned to its element), ESIZE (more than 2^30 columns), EHIP. */
int adaqp_layernorm_forward(const void *x_dev, int64_t ldx, int64_t n_rows, int32_t dim, int32_t type,
                            const float *gamma_dev, const float *beta_dev, float eps,
                            void *y_dev, int64_t ldy, float *stats_dev, void *stream);

/* Bytes of workspace adaqp_layernorm_backward needs (a multiple of 256).  Errors: EINVAL, ESIZE. */
int adaqp_layernorm_workspace_bytes(int64_t n_rows, int32_t dim, int64_t *bytes_out);

/* With h_j = (x_j - mean) * rstd and g_j = dy_j * gamma_j, for each row
 *     dx_j = rstd * (g_j - sum_i g_i / dim - h_j * sum_i g_i h_i / dim),
 * and over all rows  dgamma_j = sum dy_j h_j,  dbeta_j = sum dy_j  (zeros without rows).
 *   stats_dev      [n_rows][2] fp32, as adaqp_layernorm_forward wrote them
 *   dx_dev         NULL: not wanted; may be x or dy (same pitch)
 *   dgamma_dev, dbeta_dev   [dim] fp32, written; both NULL: not wanted (no workspace then); exactly one NULL: EINVAL
 *   workspace_dev  256-byte aligned scratch of at least adaqp_layernorm_workspace_bytes(n_rows, dim)
 * Errors: EINVAL, ESIZE (workspace too small, more than 2^30 columns), EHIP. */
int adaqp_layernorm_backward(const void *x_dev, int64_t ldx, const void *dy_dev, int64_t lddy, int64_t n_rows, int32_t dim, int32_t type,
                             const float *stats_dev, const float *gamma_dev, void *dx_dev, int64_t lddx,
                             float *dgamma_dev, float *dbeta_dev, void *workspace_dev, int64_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------------- */
/* Matrices in 4 bits.                                                                                     */
/* ---------------------------------------------------------------------------------------------------- */

/* An MX matrix of n_rows rows and n_cols columns is two arrays.
 *   codes   [n_rows][64 * ceil(n_cols / 128)] bytes: the code of column j in bits [4 (j mod 2), 4 (j mod 2) + 4) of byte j / 2 of its row.  Codes 0..7 stand
 *           for 0, 0.5, 1, 1.5, 2, 3, 4, 6, bit 3 is the sign.  Columns from n_cols on have code 0.
 *   scales  [ceil(n_cols / 128)][n_rows][4] bytes: of row r and the 32 columns 32 b .. 32 b + 31 the byte at [b / 4][r][b mod 4] = e + 127: the block's
 *           values are those of its codes times 2^e.  255: the block is NaN.
 * Both begin at a multiple of 16 bytes. */
#define ADAQP_MX4_BLOCK 32
int64_t adaqp_mx4_code_bytes(int64_t n_rows, int64_t n_cols);      /* of the two arrays; -1 for negative counts and beyond 2^62 */
int64_t adaqp_mx4_scale_bytes(int64_t n_rows, int64_t n_cols);

#define ADAQP_MX4_NEAREST 0
#define ADAQP_MX4_STOCHASTIC 1

/* Writes a matrix (x_dev [n_rows, ld] of `type`) as an MX matrix and / or its transpose as one, in one pass over x.
 * Per block (32 values of a row; for the transpose 32 values of a column; values beyond the edge count as zeros), m = the largest magnitude:
 *   NEAREST      e = floor(log2 m) - 2; each value / 2^e to the nearest of the code's values, ties to the even code, beyond 6 to 6
 *   STOCHASTIC   e = the smallest with m <= 6 * 2^e, so that nothing is clipped and the expected value is the value itself but for the 16 bits of
 *                t, which take off less than 2^-16 of hi - lo; with lo <= v / 2^e < hi the
 *                neighbours among the code's values and t = trunc(2^16 * (v / 2^e - lo) / (hi - lo)), hi is taken where t + r >= 2^16 (magnitudes; the sign
 *                stays).  r = r16(seed, row, column) of the MX matrix that is written, Philox4x32-10 as in adaqp_quantize_pack with the last
 *                counter word 0x4d583443; for the transpose seed + 1.  With e = 126 (m beyond 1.5 * 2^127) 3 stands in the place of 4: 2^128 is no
 *                fp32 number.
 * e is at least -127.  A block with an infinity or NaN: scale byte 255, codes 0.
 *   codes_dev, scales_dev       the matrix; both NULL: not wanted
 *   codes_t_dev, scales_t_dev   its transpose (n_cols rows, n_rows columns); both NULL: not wanted
 * Errors: EINVAL, ESIZE (2^31 rows or columns and more), EHIP. */
int adaqp_mx4_quantize(const void *x_dev, int64_t ld, int64_t n_rows, int64_t n_cols, int32_t type, int32_t rounding, uint64_t seed,
                       uint8_t *codes_dev, uint8_t *scales_dev, uint8_t *codes_t_dev, uint8_t *scales_t_dev, void *stream);

/* The values of an MX matrix: x_dev [n_rows, ld] of `type`, written.  All are exact; those from 2^128 on, which adaqp_mx4_quantize writes none of, are infinite.
 * Errors: EINVAL, ESIZE, EHIP. */
int adaqp_mx4_dequantize(const uint8_t *codes_dev, const uint8_t *scales_dev, int64_t n_rows, int64_t n_cols,
                         void *x_dev, int64_t ld, int32_t type, void *stream);

/* Bytes of workspace adaqp_mx4_matmul needs (a multiple of 256; 0 where the product is not split over k).  Errors: EINVAL, ESIZE. */
int adaqp_mx4_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t *bytes_out);

/* out[i, j] = sum_k a[i, k] * b[j, k]: both operands MX matrices of k columns, a of m rows, b of n rows; out_dev [m, ldo] of `type`.
 * Sums are fp32: one that passes fp32's range on its way is infinite.  With k = 0 the sum is empty and out is zeros.  A NaN block gives NaN in its row (of a) or column (of b).
 * Where few output tiles would leave the GPU idle, k is cut and the parts, held in the workspace in fp32, are added in order.
 * A layer's forward pass multiplies rows X with weights W (W's rows = outputs), its backward pass dZ with the MX form of W's transpose (giving
 * dX) and the transpose of dZ with the transpose of X (giving dW).
 * Errors: EINVAL, ESIZE (workspace too small; 2^31 rows and more; more than 2^25 columns), EHIP. */
int adaqp_mx4_matmul(const uint8_t *a_codes_dev, const uint8_t *a_scales_dev, int64_t m,
                     const uint8_t *b_codes_dev, const uint8_t *b_scales_dev, int64_t n, int64_t k,
                     void *out_dev, int64_t ldo, int32_t type, void *workspace_dev, int64_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------------------------------------------- */
/* Orthogonalised update.                                                                                  */
/* ---------------------------------------------------------------------------------------------------- */

/* Bytes of workspace adaqp_orthogonalize needs (a multiple of 256).  Errors: EINVAL, ESIZE. */
int adaqp_orthogonalize_workspace_bytes(int32_t n_matrices, int64_t n_rows, int64_t n_cols, int64_t *bytes_out);

/* For each of n_matrices matrices G of one shape:  X = G / (||G||_F + eps),  then n_steps times, with the step's (a, b, c),
 *     A = X X^T,   X <- a X + (b A + c A^2) X     (for n_rows > n_cols on the transpose, transposed back),
 * and out = X.  A step takes each singular value s to a s + b s^3 + c s^5: coefficients such as (3.4445, -4.7750, 2.0315), five times, take all that are not
 * far below the largest to about 1.
 *   g_dev, out_dev   matrix i at g + i * stride_g and out + i * stride_o (elements), pitches ldg and ldo; out may be g (same pitch and stride)
 *   coef_host        [n_steps][3], host memory, read during the call
 * The norm is summed in 64 bits.  Products are taken on the matrix cores with every operand held as the sum of two fp16 numbers (22 bits), which
 * need a bound on it: the coefficients must keep singular values from [0, 1] below ADAQP_ORTHOGONALIZE_MOST at every step, else EINVAL.  Matrices with
 * infinities or NaN give NaN throughout.
 * Errors: EINVAL, ESIZE (workspace too small, more than 65535 matrices, 2^20 rows or columns and more), EHIP. */
#define ADAQP_ORTHOGONALIZE_MOST 4.0
int adaqp_orthogonalize(const void *g_dev, int64_t ldg, int64_t stride_g, void *out_dev, int64_t ldo, int64_t stride_o,
                        int32_t n_matrices, int64_t n_rows, int64_t n_cols, int32_t type, int32_t n_steps, const float *coef_host, float eps,
                        void *workspace_dev, int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ADAQP_DENSE_H */
