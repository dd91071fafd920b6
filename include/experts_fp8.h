/* experts_fp8 -- matrix products of 8-bit floating-point operands with a scale for each block of 128 values, and what
 * routes tokens to experts around them, on MI355X (gfx950).  The floating-point sibling of gemm_int8_nt and of the
 * requantising activation in conv2d_int8.h; same library, same conventions:
 *   - Every pointer is a DEVICE pointer owned by the caller; the library never frees or keeps it.  `stream` is a
 *     hipStream_t passed as void* (NULL = the default stream).  All work is enqueued on it; no call synchronises with the
 *     host, allocates, or needs a workspace, so every call may be captured into a HIP graph.
 *   - Every function returns a conv_status_t.  Arguments are validated before anything is enqueued.  Nothing throws.
 *     What only the device holds (ids, offsets, rows) is bounded by the kernels: a value out of range is no index.
 *     Products whose extents pass 2^30 - 1 (summed ones 2^31 - 256) or whose results reach 2^24 tiles of 128 x 128 are
 *     CONV_ERR_UNSUPPORTED, as are over 2^25 - 4 tokens of a routing or pairs or rows of a combination's backward pass.
 *   - Matrices are row-major; ld* is the distance of two rows in ELEMENTS, at least the row's length.  Any extent may be
 *     0 unless stated (nothing is read, results of an empty sum are zeros).
 *   - 8-bit values are OCP e4m3 (largest 448, no infinity).  Operands whose rows begin on 16 bytes are read fastest; any
 *     other alignment and any length are read, more slowly.
 */
#ifndef EXPERTS_FP8_H
#define EXPERTS_FP8_H

#include "conv2d_int8.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    EXPERTS_F32 = 0,
    EXPERTS_BF16 = 1,
    EXPERTS_F16 = 2
} experts_type_t;

#define EXPERTS_BLOCK 128        /* values to a scale */
#define EXPERTS_MOST 1024        /* experts of one routing */
#define EXPERTS_MOST_CHOICES 64  /* experts of one token */

/* ---- quantisation -----------------------------------------------------------------------------------------------
 * q = rne_e4m3(clamp(x / scale, -448, 448)), scale = the least power of two >= (largest finite |x| of the block) / 448,
 * from 2^-126 on; 1 for a block of zeros.  A power of two: the division is exact and so is what the products multiply back.
 * An infinity becomes +-448, a NaN stays one and does not count for the scale.
 * gate != 0: x = silu(first cols columns) * (next cols columns) of the source (2 * cols columns), in 32 bits.
 * take (may be NULL): int32 [rows]; row r of x is source row take[r] / per_row, zeros where take[r] is negative or past
 * src_rows * per_row (the order of expert_rows; without it the source has `rows` rows).
 * quantize_fp8_rows   q [rows][cols], a scale for 128 columns of a row: scales [ceil(cols/128)][rows]
 * quantize_fp8_columns   qt [cols][rows], a scale for 128 rows of a column: scales_t [ceil(rows/128)][cols]; and, where q is
 *     not NULL, what quantize_fp8_rows gives as well, from the same read
 * quantize_fp8_tiles  count matrices [rows][cols], each at src + i * rows * lds and q + i * (its rows) * ldq: a scale for 128 x 128;
 *     transpose == 0: q [rows][cols], scales [ceil(rows/128)][ceil(cols/128)]; != 0: both transposed
 * Scales are dense.  A launch takes rows of up to 2^30 - 1 and 2^24 - 1 pieces of 128 x 128, or of 16 rows x 512 columns (quantize_fp8_rows); more:
 * CONV_ERR_UNSUPPORTED. */
int quantize_fp8_rows(int rows, int cols, const void *src, int type, long long lds, int gate, const int32_t *take, int per_row, int src_rows,
                      uint8_t *q, long long ldq, float *scales, void *stream);
int quantize_fp8_columns(int rows, int cols, const void *src, int type, long long lds, int gate, const int32_t *take, int per_row, int src_rows,
                         uint8_t *qt, long long ldqt, float *scales_t, uint8_t *q, long long ldq, float *scales, void *stream);
int quantize_fp8_tiles(int count, int rows, int cols, const void *src, int type, long long lds, int transpose,
                       uint8_t *q, long long ldq, float *scales, void *stream);
/* Gradient of silu(g) * u:  x [rows][2 * cols] holds g and u, dh [rows][cols] -> dx [rows][2 * cols], all of one type. */
int silu_gate_backward(int rows, int cols, const void *x, long long ldx, const void *dh, long long ldh, void *dx, long long lddx, int type, void *stream);

/* ---- products ------------------------------------------------------------------------------------------------------
 * C[m][n] = sum over blocks b of 128 of K:  sa[b][m] * sb * (sum over k in b of A[m][k] * B[n][k]), 32-bit sums,
 * rounded once to out_type.  A [M][K], sa [ceil(K/128)][M] dense.  b_rows == 0: sb[n / 128][b] ([ceil(N/128)][ceil(K/128)], weights);
 * != 0: sb[b][n] ([ceil(K/128)][N]).  Scales are any f32 whose products sa * sb are finite too.  Gradients are the same product: of the
 * input with the weights quantised transposed, of the weights with both operands quantised by columns.
 * fast_sums != 0: the sum within a block may be taken by the 8-bit matrix instruction, up to twice as fast, which cuts each of eight
 * neighbouring products (k = 8 i ... 8 i + 7) towards zero to a multiple of 2^-13 of the largest one's power of two.  A result is then up
 * to 7 * 2^-13 (8.5e-4) of the sum of its terms' magnitudes off, which is more than rounding to float16; with values of one size and random
 * sign 1.5e-5 of the result in the mean, a hundredth of rounding to bfloat16, but losses of terms of one sign add up. */
int gemm_fp8_nt(int M, int N, int K, const uint8_t *A, long long lda, const float *sa, const uint8_t *B, long long ldb, const float *sb, int b_rows,
                void *C, long long ldc, int out_type, int fast_sums, void *stream);
/* A weight matrix for each expert.  Row r of C, offsets[e] <= r < offsets[e + 1], is the product of A's row r -- with rows
 * (int32 [R]) of A's row rows[r] / per_row -- and W + e * N * ldw (scales at sw + e * ceil(N/128) * ceil(K/128)).  Rows that
 * belong to no expert (ahead of offsets[0], from offsets[E] on), and those whose rows[r] is negative or past a_rows * per_row, are zeros.  offsets: int32
 * [E + 1], rising, within 0 to R.  A [a_rows][K] (a_rows = R without rows), sa [ceil(K/128)][a_rows]; E up to EXPERTS_MOST. */
int gemm_fp8_experts(int R, int a_rows, int E, int N, int K, const uint8_t *A, long long lda, const float *sa, const uint8_t *W, long long ldw,
                     const float *sw, const int32_t *offsets, const int32_t *rows, int per_row, void *C, long long ldc, int out_type, int fast_sums, void *stream);
/* Their weights' gradients: C[e][n][k] = sum over r in [offsets[e], offsets[e + 1]) of A[n][r] * B[k][r], with A [N][R], sa
 * [ceil(R/128)][N], B [K][R], sb [ceil(R/128)][K]: both operands quantised by columns.  C + e * N * ldc.  Offsets of
 * multiples of 128 (expert_rows with align 128) are fastest. */
int gemm_fp8_experts_grad(int R, int E, int N, int K, const uint8_t *A, long long lda, const float *sa, const uint8_t *B, long long ldb, const float *sb,
                          const int32_t *offsets, void *C, long long ldc, int out_type, int fast_sums, void *stream);

/* ---- routing ----------------------------------------------------------------------------------------------------------
 * s = softmax(logits) (sigmoid != 0: 1 / (1 + exp(-logits))) over a token's E experts; an expert whose logit is -infinity or NaN
 * is not to be had and has no part in the softmax; +infinity counts as the largest finite value.  Choice by c = s + bias
 * (bias: f32 [E] or NULL; an expert whose c is -infinity or NaN is not to be had): of `groups` equal
 * groups of neighbouring experts the `kept` of highest score (the sum of the group_top (1 or 2) largest c of those to be had, the lowest finite number at least) remain, of their
 * experts the k of largest c, in falling order; ties go to the lower index.  ids [T][k] int32, -1 where fewer are to be had.
 * weights [T][k] f32: s of the chosen (without the bias), / (their sum + 1e-20) if renormalise, * factor; 0 beside -1.
 * E up to EXPERTS_MOST, k up to EXPERTS_MOST_CHOICES and to E, groups up to 64. */
int route_experts(int T, int E, int k, const void *logits, int type, long long ldl, const float *bias, int sigmoid, int groups, int kept, int group_top,
                  int renormalise, float factor, int32_t *ids, float *weights, void *stream);
/* dlogits [T][E] (the logits' type) from dweights [T][k] f32 and the ids of route_experts. */
int route_experts_backward(int T, int E, int k, const void *logits, int type, long long ldl, const int32_t *ids, const float *dweights, int sigmoid,
                           int renormalise, float factor, void *dlogits, long long lddl, void *stream);
/* Order of the experts' rows: the pairs p = t * k + j of ids [pairs] sorted by expert, in their own order within one.
 * offsets [E + 1]: expert e's rows are offsets[e] ... offsets[e + 1] - 1, its pairs first; every offset is a multiple of
 * align (1 to 1024).  rows [R]: the pair of a row, -1 where there is none.  place [pairs]: the row of a pair, -1 for an id that
 * is no expert.  R is expert_rows_capacity(pairs, E, align) (0: invalid). */
int expert_rows_capacity(int pairs, int E, int align);
int expert_rows(int pairs, int E, int align, const int32_t *ids, int32_t *offsets, int32_t *rows, int32_t *place, void *stream);

/* ---- combination -----------------------------------------------------------------------------------------------------
 * out[t] = sum over j of weights[t][j] * y[place[t][j]], 32-bit sums; y [R][N]; weights f32 [T][k] or NULL for ones;
 * a place that is no row of y adds nothing.  out and y of one type, out of up to 2^40 numbers (more: CONV_ERR_UNSUPPORTED). */
int combine_experts(int T, int k, int N, int R, const void *y, long long ldy, int type, const int32_t *place, const float *weights,
                    void *out, long long ldo, void *stream);
/* dy[r] = weights[p] * dout[p / k] for the pair p = rows[r] with place[p] = r, zeros for a row of no pair; dweights[p] = dout[p / k] . y[place[p]],
 * 0 for a pair of no row.  dout [T][N], dy [R][N] of y's type. */
int combine_experts_backward(int T, int k, int N, int R, const void *dout, long long ldd, const void *y, long long ldy, int type, const int32_t *place,
                             const int32_t *rows, const float *weights, void *dy, long long lddy, float *dweights, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* EXPERTS_FP8_H */
