/*
 * mxfp8_b128.h -- C ABI of FP8 operands with an FP32 scale for each block of 128: the coarser-grained recipe beside MXFP8 (blocks
 * of 32, power-of-two scales). Same library and conventions as mxfp8.h: device pointers, the caller owns every buffer, nothing is
 * allocated, kept or synchronised, work goes to `hip_stream`, errors by return code before any launch. No output overlaps an
 * input or another output.
 *
 *   training  mxfp8_b128_quantize(X, MXFP8_BOTH, VECTORS)     X_row, X_colT    (dY the same)
 *             mxfp8_b128_quantize(W, MXFP8_BOTH, TILES)       W_row, W_colT
 *             mxfp8_b128_gemm(MXFP8_FPROP)  Y  = X_row   * W_row^T
 *             mxfp8_b128_gemm(MXFP8_DGRAD)  dX = dY_row  * W_colT^T
 *             mxfp8_b128_gemm(MXFP8_WGRAD)  dW = dY_colT * X_colT^T
 *   serving   mxfp8_b128_quantize(W, MXFP8_ROWWISE, TILES) once, mxfp8_b128_gemv for a few rows of BF16 activations
 *             (mxfp8_expert_layer of mxfp8_layer.h for experts)
 *
 * An operand [rows x cols] is E4M3 bytes with a leading dimension `ld`, a multiple of 16, and FP32 scales. It is cut into
 *   VECTORS  blocks of 128 consecutive columns of a row; the scale of block b of row r is s[b * rows + r]
 *   TILES    blocks of 128 x 128; the scale of rows 128 i .. and columns 128 j .. is s[i * ceil(cols / 128) + j]
 * Blocks at the end may be shorter. Where cols is not a multiple of 16, the bytes of a row up to the next multiple of 16 belong
 * to the operand (in the last row too) and are zero.
 */
#ifndef MXFP8_B128_H
#define MXFP8_B128_H

#include "mxfp8.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { MXFP8_B128_VECTORS = 0, MXFP8_B128_TILES = 1 } mxfp8_b128_shape;

/*
 * Converts src [rows x cols] (FP32 or BF16, leading dimension ld_src >= cols):
 *   X   = largest magnitude of the block / 448, rounded to FP32; at least 2^-126
 *   Q_i = V_i / X, rounded to FP32 and then to E4M3 (both to nearest even)
 * into an operand [rows x cols] in q_row, s_row (MXFP8_ROWWISE), the transposed operand [cols x rows] in q_colT, s_colT
 * (MXFP8_COLWISE), or both from one read. VECTORS: the blocks of the transposed operand are 128 rows of a column of src, converted
 * from src itself. TILES: both hold the same codes, the scales of the transposed one are transposed.
 * The padding bytes of the rows are written (zeros). A block with a NaN gets the scale NaN and codes 0x7F. A block with an infinity and no
 * NaN counts FLT_MAX as its largest magnitude: infinities become +-448. The sign of every input, zero included, is kept.
 * Any rows and cols up to 2^30, up to 2^31 - 1 tiles of 128 x 128; src aligned to its element size (faster: it and its rows
 * 16-byte aligned), q_row and q_colT 16-byte aligned, ld_row >= cols and ld_colT >= rows multiples of 16, scales 4-byte aligned.
 * Outputs that `axis` does not select are ignored and may be NULL.
 */
mxfp8_status mxfp8_b128_quantize(const void *src, mxfp8_dtype src_dtype, int64_t rows, int64_t cols, int64_t ld_src,
                                 mxfp8_axis axis, mxfp8_b128_shape shape, uint8_t *q_row, int64_t ld_row, float *s_row,
                                 uint8_t *q_colT, int64_t ld_colT, float *s_colT, void *hip_stream);

/* Bytes of workspace of mxfp8_b128_gemm (host arithmetic); 0 where it needs none, -1 for sizes it does not take or an unknown pass. */
int64_t mxfp8_b128_gemm_workspace(mxfp8_pass pass, int64_t M, int64_t N, int64_t K);

/*
 * C [M x N] = A [M x K] * B [N x K]^T: C[m, n] = sum over blocks b of a_s * b_s * sum over k in b of A[m, k] B[n, k], each block's sum
 * on the matrix instructions, scaled and added up in FP32. The type of c chooses how a block's sum is made: for BF16 by the FP8 instructions,
 * which cut every product of eight neighbours off at 2^-13 of the largest of them (below the result's rounding); for FP32 from the
 * codes widened to BF16, exactly, with FP32 additions, at half the rate. A is cut into VECTORS; B into TILES in MXFP8_FPROP and
 * MXFP8_DGRAD, into VECTORS in MXFP8_WGRAD (the operand table above). The product of two scales is formed in FP32, before the block's sum is
 * multiplied with it: one beyond its range counts as infinite, one below 2^-126 as a subnormal.
 * c FP32 or BF16 (rounded to nearest even), leading dimension ldc >= N, aligned to its element size (faster: c and its rows
 * 16-byte aligned). Any M, N up to 2^30 and K up to 2^24, ceil(M / 32) * ceil(N / 32) < 2^31 (otherwise MXFP8_ERR_SHAPE); K == 0 stores
 * zeros. a_q, b_q 16-byte aligned, lda, ldb multiples of 16 below 2^24 + 16; scales 4-byte aligned.
 * workspace: mxfp8_b128_gemm_workspace bytes, 16-byte aligned, contents meaningless before and after (the sums of parts of K, where
 * there are few tiles); calls that may run at the same time, captured graphs among them, need one each.
 * A NaN in an element or a scale makes every output that it touches NaN. The order of the sums depends on the sizes and the type of c alone.
 */
mxfp8_status mxfp8_b128_gemm(mxfp8_pass pass, const uint8_t *a_q, int64_t lda, const float *a_s, const uint8_t *b_q, int64_t ldb,
                             const float *b_s, int64_t M, int64_t N, int64_t K, void *c, mxfp8_dtype c_dtype, int64_t ldc,
                             void *workspace, void *hip_stream);

/*
 * C [M x N] = x [M x K] * W [N x K]^T for a few rows of BF16 activations and weights cut into TILES: codes are widened to BF16
 * (exactly), multiplied with the activations as they are, a block's sum is scaled and added up in FP32. c as above, leading
 * dimension ldc >= N. Meant for up to some thirty rows, where reading the weights is all the work; any M is right. K % 16 == 0, K <= 2^24,
 * M, N <= 2^30, ceil(N / 16) * M < 2^23 (products of many rows are taken up to 16 times that, then MXFP8_ERR_SHAPE); x 16-byte
 * aligned, ldx a multiple of 8; w_q 16-byte aligned, ldw >= K a multiple of 16; w_s 4-byte aligned; c aligned to its element size.
 */
mxfp8_status mxfp8_b128_gemv(const void *x_bf16, int64_t ldx, const uint8_t *w_q, int64_t ldw, const float *w_s, int64_t M,
                             int64_t N, int64_t K, void *c, mxfp8_dtype c_dtype, int64_t ldc, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MXFP8_B128_H */
