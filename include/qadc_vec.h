/*
 * qadc_vec.h -- operators on the vectors that libqadc searches: where they come from (rows of a table, looked up by
 * id, and the gradient that trains it), the root-mean-square norm in front of a projection, and products of 8-bit
 * matrices with a scale for each block of 128 values (the projection itself, its gradients, or the scores of queries
 * against vectors kept in 8 bits).
 *
 * The conventions of qadc.h hold: [dev] pointers are the caller's, every call only enqueues work on `stream`, nothing
 * is allocated, 0 or a negative code comes back and pq_last_error() says what was wrong.  Beyond them:
 *   - Matrices are row-major; `ld_x` is the distance of two rows of x in elements, at least the number of columns.  No
 *     alignment beyond that of the element is needed; rows that start at multiples of 16 bytes are read fastest.
 *   - Only the named elements are read or written, never the space between rows.
 *   - Values are finite or not: infinities and NaN give what the formulas give.  Sums are in float32 and in a fixed
 *     order: two calls with the same arguments give the same bits.
 *   - Outputs must not overlap inputs, except where a call says so.
 *   - Results are rounded once to the output's type, to nearest, ties to even.
 */
#ifndef QADC_VEC_H
#define QADC_VEC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element types.  E4M3 (no infinity, largest 448) and E5M2 (largest 57344) are the 8-bit floats; E8M0 is a power of two
 * 2^(byte - 127), byte 255 being NaN. */
enum { VEC_F32 = 0, VEC_BF16 = 1, VEC_F16 = 2, VEC_E4M3 = 3, VEC_E5M2 = 4, VEC_E8M0 = 5 };

#define VEC_BLOCK 128         /* consecutive values that share a scale */
#define VEC_MAX_NORM_DIM 16384 /* columns of vec_norm and vec_norm_grad */
#define VEC_MAX_ROW_DIM (1 << 24) /* columns of vec_lookup and vec_lookup_grad */

/*
 * out[i] = scale * table[ids[i]].  An id outside 0..rows-1 (a search pads its results with -1) gives a row of zeros.
 *   table [dev][rows][d], table_type F32, BF16 or F16; rows >= 0, 1 <= d <= VEC_MAX_ROW_DIM
 *   ids   [dev][n], int32 (id_bytes 4) or int64 (8); n >= 0
 *   out   [dev][n][d], out_type F32, BF16 or F16
 */
int vec_lookup(const void *table, int64_t rows, int d, int64_t ld_table, int table_type, const void *ids, int id_bytes,
               int64_t n, float scale, void *out, int64_t ld_out, int out_type, void *stream);

/*
 * The gradient of vec_lookup for its table:
 *   table_grad[v] = (accumulate ? table_grad[v] : 0) + scale * sum over the i with ids[i] == v of grad[i]
 * Every row is written, those without an id with zeros (accumulate: these are left alone).  Ids outside 0..rows-1 take no part.
 *   grad       [dev][n][d], grad_type F32, BF16 or F16; n < 2^31, 1 <= d <= VEC_MAX_ROW_DIM
 *   table_grad [dev][rows][d], table_type F32, BF16 or F16; rows < 2^31
 *   workspace  >= vec_lookup_grad_workspace_bytes(n, rows, d), 256-byte aligned, any content
 */
size_t vec_lookup_grad_workspace_bytes(int64_t n, int64_t rows, int d);
int vec_lookup_grad(const void *grad, int64_t n, int d, int64_t ld_grad, int grad_type, const void *ids, int id_bytes,
                    float scale, int accumulate, void *table_grad, int64_t rows, int64_t ld_table, int table_type,
                    void *workspace, size_t workspace_bytes, void *stream);

/*
 * Root-mean-square norm of every row, with the addition that feeds it and an 8-bit result:
 *   h = x + residual, rounded to the type (x itself without a residual)
 *   y = h / sqrt(mean(h^2) + eps) * weight                                             (float32)
 *   q, scales = the blocks of y as vec_quantize_blocks makes them from float32 values
 * x, residual, h and y are [dev][n][d] of one type (F32, BF16 or F16), weight is [dev][d] (weight_type: that type or F32).
 *   residual, h  both or neither; h may be x or residual itself (same pointer and ld)
 *   y            or NULL           q, scales  both or neither; not both y and q NULL
 * 1 <= d <= VEC_MAX_NORM_DIM, eps >= 0.
 */
int vec_norm(const void *x, int64_t ld_x, const void *residual, int64_t ld_residual, int type, const void *weight,
             int weight_type, int64_t n, int d, float eps, void *h, int64_t ld_h, void *y, int64_t ld_y, void *q,
             int64_t ld_q, int q_type, void *scales, int64_t ld_scales, int scale_type, void *stream);

/*
 * The gradient of vec_norm.  dy is the gradient of y (or of q * scales: the rounding to 8 bits counts as the identity);
 * h is what vec_norm returned (x where it had no residual).  With u = dy * weight and r = 1 / sqrt(mean(h^2) + eps):
 *   dx      = r * u - h * r^3 * mean(u * h) + dh      the gradient of x, and the same of residual
 *   dweight = sum over the rows of dy * h * r         [dev][d] float32
 *   dh      the gradient that reaches h past the norm, or NULL
 * dy, h, dh and dx are of one type; dx may be dh or dy itself (same pointer and ld).
 *   workspace >= vec_norm_grad_workspace_bytes(n, d), 256-byte aligned, any content
 */
size_t vec_norm_grad_workspace_bytes(int64_t n, int d);
int vec_norm_grad(const void *dy, int64_t ld_dy, const void *h, int64_t ld_h, const void *dh, int64_t ld_dh, int type,
                  const void *weight, int weight_type, int64_t n, int d, float eps, void *dx, int64_t ld_dx, float *dweight,
                  void *workspace, size_t workspace_bytes, void *stream);

/*
 * 8-bit values with a scale for each block of VEC_BLOCK of them.  With a the largest finite magnitude of the block and
 * L the largest value of q_type (448 or 57344):
 *   scale = E8M0: the smallest power of two with a <= L * scale, at least 2^-127
 *           F32:  a / L, at least 2^-126          1 where a = 0
 *   q     = the float32 quotient x / scale, rounded to q_type; NaN, and infinity in E4M3, become NaN
 *   x [dev][n][d] of type F32, BF16 or F16; n ceil(d / 128) < 2^35
 *   transposed == 0: blocks run along a row:   q [dev][n][d], scales [dev][n][ceil(d / 128)]
 *   transposed == 1: blocks run along a column, and the result is transposed (the factors of a weight gradient):
 *                                              q [dev][d][n], scales [dev][d][ceil(n / 128)]
 */
int vec_quantize_blocks(const void *x, int64_t ld_x, int type, int64_t n, int64_t d, int transposed, void *q, int64_t ld_q,
                        int q_type, void *scales, int64_t ld_scales, int scale_type, void *stream);

/*
 * c[i][j] = sum over k of (a[i][k] * a_scales[i][k / 128]) * (b[j][k] * b_scales[j][k / 128])
 *   a [dev][m][k], b [dev][n][k] of type E4M3 or E5M2 (each its own); both scales of scale_type E8M0 or F32
 *   c [dev][m][n] of c_type F32, BF16 or F16
 * Products are exact and their sums are in float32.  E8M0 scales are applied to the values (what is below 2^-126 may then count as zero); F32
 * scales to each block's sum, by the product of the two in float32 (2^-126 to 2^128: beyond it the sum loses bits, or is 0, infinite or NaN).
 * k == 0 gives zeros.  m, n, k < 2^31, and with m > 32 less than 2^24 tiles of 128 x 128 of c.
 *   workspace >= vec_matmul_blocks_workspace_bytes(m, n, k) (may be 0), 256-byte aligned, any content
 */
size_t vec_matmul_blocks_workspace_bytes(int64_t m, int64_t n, int64_t k);
int vec_matmul_blocks(const void *a, int64_t ld_a, int a_type, const void *a_scales, int64_t ld_a_scales, const void *b,
                      int64_t ld_b, int b_type, const void *b_scales, int64_t ld_b_scales, int scale_type, int64_t m,
                      int64_t n, int64_t k, void *c, int64_t ld_c, int c_type, void *workspace, size_t workspace_bytes,
                      void *stream);

#ifdef __cplusplus
}
#endif
#endif /* QADC_VEC_H */
