/*
 * mxfp8_experts.h -- C ABI of what surrounds the products of a mixture-of-experts layer (Appendix A.4: the recipe applies unchanged
 * to the expert products), and of products of a few rows with MXFP4 weights. Same library and conventions as mxfp8.h: device
 * pointers, the caller owns every buffer, nothing is allocated, kept or synchronised, work goes to `hip_stream`, errors by
 * return code before any launch. No output overlaps an input or another output.
 *
 *   training  mxfp8_expert_sort(experts, align = 128)                       plan
 *             mxfp8_expert_quantize_ex(x, no weights, MXFP8_BOTH)           X_row, X_colT of the sorted rows
 *             mxfp8_gemm_grouped_ex(MXFP8_FPROP)                            C [rows x N]
 *             mxfp8_expert_combine(C, weights)                              y [tokens x N]
 *   backward  mxfp8_expert_weight_grad(dy, C)                               dweights [tokens x slots]
 *             mxfp8_expert_quantize_ex(dy, weights, MXFP8_BOTH)             dC_row, dC_colT
 *             mxfp8_gemm_grouped_ex(MXFP8_DGRAD, MXFP8_WGRAD)               dX of the sorted rows, dW of each expert
 *             mxfp8_expert_combine(dX, no weights)                          dx [tokens x K]
 *   serving   mxfp8_expert_sort(align = 1), mxfp8_fp4_gemv_grouped_ex, mxfp8_expert_combine
 *
 * A token chooses `slots` experts. ENTRY i = t * slots + j stands for slot j of token t; there are entries = tokens * slots.
 */
#ifndef MXFP8_EXPERTS_H
#define MXFP8_EXPERTS_H

#include "mxfp8.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { MXFP8_I32 = 0, MXFP8_I64 = 1 } mxfp8_index;

/* Rows that sorted entries take at most: entries + min(entries, groups) * (align - 1), cut down to a multiple of align (host
 * arithmetic). -1 for entries outside [0, 2^30], groups outside [0, 4096], an align that is not a power of two up to 4096, or
 * more than 2^30 rows. */
int64_t mxfp8_expert_rows(int64_t entries, int32_t groups, int32_t align);

/* Bytes of workspace of mxfp8_expert_sort (host arithmetic); 0 where it needs none, -1 for sizes as above. */
int64_t mxfp8_expert_sort_workspace(int64_t entries, int32_t groups);

/*
 * Sorts the entries by expert, keeping their order within an expert, each expert's rows padded to a multiple of `align`:
 *   experts     [entries] int32 or int64; anything outside [0, groups) has no expert
 *   positions   [entries] int32: the entry's row, -1 without an expert
 *   sources     [rows] int32: the row's entry, -1 for rows of the padding and behind the last expert
 *   group_ends  [groups] int32: the padded ends of the experts' rows, as mxfp8_gemm_grouped_ex wants them (align 64 for
 *               tiled scales, 128 for the weight gradient)
 * rows >= mxfp8_expert_rows(entries, groups, align). workspace: mxfp8_expert_sort_workspace bytes, contents meaningless before
 * and after; calls that may run at the same time, captured graphs among them, need one each. experts 8- or 4-byte aligned as their
 * type, workspace and the outputs 4-byte aligned; nothing overlaps.
 */
mxfp8_status mxfp8_expert_sort(const void *experts, mxfp8_index experts_type, int64_t entries, int32_t groups, int32_t align,
                               int64_t rows, int32_t *positions, int32_t *sources, int32_t *group_ends, void *workspace,
                               void *hip_stream);

/*
 * MXFP8 copies of sorted rows: what mxfp8_quantize_ex makes of the tensor v [rows x cols]
 *   v[r, :] = weights[i] * src[i / slots, :] with i = sources[r]  (without weights: src[i / slots, :])
 *   v[r, :] = 0 where sources[r] is -1
 * which is never stored. The product with the weight is rounded once, by the conversion (a product below 2^-102 may have been
 * rounded to FP32 before; one beyond FP32 counts as infinite). src [tokens x cols] FP32 or BF16, leading dimension
 * ld_src; weights [tokens x slots] FP32, NULL for none; group_ends [groups] as mxfp8_expert_sort gave them: rows behind the last
 * 128-row tile that holds a row of an expert are left as they were (NULL with groups == 0: all rows are converted). An entry number
 * outside [-1, tokens * slots) counts as -1 and an end outside [0, rows] as the nearer of the two, so that no access leaves a buffer.
 * Elements, scales, axes, outputs and their layouts as mxfp8_quantize_ex (E4M3, scales rounded up). rows % 32 == 0, cols % 32 ==
 * 0; src 16-byte aligned, ld_src a multiple of 16 bytes; q_row, q_colT and tiled scales 16-byte aligned; sources, weights,
 * group_ends 4-byte aligned; tokens <= 2^30, slots in [1, 4096], tokens * slots <= 2^30.
 */
mxfp8_status mxfp8_expert_quantize_ex(const void *src, mxfp8_dtype src_dtype, int64_t tokens, int64_t cols, int64_t ld_src,
                                      const int32_t *sources, int32_t slots, const float *weights, const int32_t *group_ends,
                                      int32_t groups, int64_t rows, mxfp8_axis axis, uint8_t *q_row, uint8_t *s_row,
                                      uint8_t *q_colT, uint8_t *s_colT, mxfp8_scale_layout scale_layout, void *hip_stream);

/*
 * Sorted rows back to their tokens: out[t, :] = sum over j of weights[t, j] * c[positions[t, j], :] (without weights: the plain
 * sum, which is the gradient of the sorted copies), summed in FP32 in the order of j and rounded once. A position outside
 * [0, rows) adds nothing, whatever its weight; a token without any gets zeros. c [rows x cols] and out [tokens x cols] FP32 or
 * BF16, leading dimensions ldc, ld_out; positions [tokens x slots]; weights [tokens x slots] FP32 or NULL. Any cols; c and out aligned
 * to their element size (faster: cols % 8 == 0, they and their rows 16-byte aligned); positions and weights 4-byte aligned. Sizes as above, and
 * tokens * ceil(cols / 512) < 2^31.
 */
mxfp8_status mxfp8_expert_combine(const void *c, mxfp8_dtype c_dtype, int64_t rows, int64_t cols, int64_t ldc,
                                  const int32_t *positions, const float *weights, int64_t tokens, int32_t slots, void *out,
                                  mxfp8_dtype out_dtype, int64_t ld_out, void *hip_stream);

/*
 * Gradient of mxfp8_expert_combine for its weights: dweights[t, j] = sum over columns of dy[t, :] * c[positions[t, j], :], in FP32;
 * 0 for a position outside [0, rows). dy [tokens x cols], c [rows x cols] FP32 or BF16, dweights [tokens x slots] FP32 dense. The
 * order of the sum depends on the sizes alone. Requirements as for mxfp8_expert_combine, dy in the place of out; dweights 4-byte
 * aligned.
 */
mxfp8_status mxfp8_expert_weight_grad(const void *dy, mxfp8_dtype dy_dtype, int64_t ld_dy, const void *c, mxfp8_dtype c_dtype,
                                      int64_t rows, int64_t cols, int64_t ldc, const int32_t *positions, int64_t tokens,
                                      int32_t slots, float *dweights, void *hip_stream);

/*
 * C [M x N] = x [M x K] * W [N x K]^T for a few rows of BF16 activations and MXFP4 weights as mxfp8_fp4_quantize_ex stores them
 * (w_q [N x K/2], w_s [N x K/32] in `scale_layout`): the weights are widened to BF16, as mxfp8_fp4_dequantize_ex gives them, on their
 * way to the matrix instructions and accumulated in FP32; activations are not quantized. c FP32 or BF16 (RNE), leading dimension
 * ldc >= N. Meant for up to some thirty rows, where reading the weights is all the work; any M is right. M, N <= 2^30, K <= 2^24,
 * ceil(N / 16) * M < 2^23 (products of many rows are taken up to 32 times that, then MXFP8_ERR_SHAPE); K % 32 == 0 (K == 0 stores
 * zeros); x 16-byte aligned and ldx a multiple of 8; w_q and tiled w_s 16-byte aligned; c aligned to its element size (faster: c and
 * its rows 16-byte aligned). A 0xFF scale makes its output column NaN.
 */
mxfp8_status mxfp8_fp4_gemv_ex(const void *x_bf16, int64_t ldx, const uint8_t *w_q, const uint8_t *w_s, int64_t M, int64_t N,
                               int64_t K, void *c, mxfp8_dtype c_dtype, int64_t ldc, mxfp8_scale_layout scale_layout,
                               void *hip_stream);

/*
 * The same for the rows of a plan, each with its expert's weights: row r of C, for r below group_ends[groups - 1], is
 * x[sources[r] / slots, :] * W_e^T for the expert e that owns r, zeros where sources[r] is -1; later rows are left as they
 * were. x [tokens x K]; sources [M]; w_q [groups x N x K/2]; expert e's scales start mxfp8_scale_bytes(N, K, scale_layout) bytes after
 * e-1's. sources may be NULL: row r takes x[r] (M <= tokens; slots is not looked at), as the second product of an expert needs.
 * Entry numbers outside [-1, tokens * slots) count as -1, ends are clamped to [0, M]; ends that decrease give undefined values.
 * groups <= 4096; sources and group_ends 4-byte aligned; everything else as above.
 */
mxfp8_status mxfp8_fp4_gemv_grouped_ex(const void *x_bf16, int64_t tokens, int64_t ldx, const int32_t *sources, int32_t slots,
                                       const uint8_t *w_q, const uint8_t *w_s, const int32_t *group_ends, int32_t groups,
                                       int64_t M, int64_t N, int64_t K, void *c, mxfp8_dtype c_dtype, int64_t ldc,
                                       mxfp8_scale_layout scale_layout, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MXFP8_EXPERTS_H */
