// Launches of the expert rows and of the MXFP4 products of a few rows; arguments as the entry points have checked them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mxfp8 {
int64_t expert_sort_workspace(int64_t entries, int groups);
hipError_t launch_expert_sort(const void *experts, bool index64, int64_t entries, int groups, int align, int64_t rows, int32_t *positions,
                              int32_t *sources, int32_t *group_ends, uint32_t *workspace, hipStream_t stream);
hipError_t launch_expert_quantize(const void *src, bool bf16, int64_t tokens, int64_t cols, int64_t ld, const int32_t *sources, int slots,
                                  const float *weights, const int32_t *group_ends, int groups, int64_t rows, int axis, uint8_t *q_row,
                                  uint8_t *s_row, uint8_t *q_colT, uint8_t *s_colT, bool tiled_scales, hipStream_t stream);
hipError_t launch_expert_combine(const void *c, bool c_bf16, int64_t rows, int64_t cols, int64_t ldc, const int32_t *positions,
                                 const float *weights, int64_t tokens, int slots, void *out, bool out_bf16, int64_t ld_out, hipStream_t stream);
hipError_t launch_expert_weight_grad(const void *dy, bool dy_bf16, int64_t ld_dy, const void *c, bool c_bf16, int64_t rows, int64_t cols,
                                     int64_t ldc, const int32_t *positions, int64_t tokens, int slots, float *dw, hipStream_t stream);
hipError_t launch_fp4_gemv(const void *x, int64_t tokens, int64_t ldx, const int32_t *sources, int slots, const uint8_t *w_q, const uint8_t *w_s,
                           const int32_t *group_ends, int groups, int64_t ws_group_bytes, int64_t M, int64_t N, int64_t K, void *c, bool c_bf16,
                           int64_t ldc, bool tiled_scales, hipStream_t stream);
}  // namespace mxfp8
