// C ABI of the expert rows and of the MXFP4 products of a few rows (include/mxfp8_experts.h): argument validation on the host, then
// the call's kernels on the caller's stream.
#include "../../include/mxfp8_experts.h"

#include "expert_launches.h"

namespace {
inline bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline bool valid_dtype(int d) { return d == MXFP8_F32 || d == MXFP8_BF16; }
inline bool valid_layout(int l) { return l == MXFP8_SCALES_ROWMAJOR || l == MXFP8_SCALES_TILED; }
inline int64_t esize(int d) { return d == MXFP8_BF16 ? 2 : 4; }
inline mxfp8_status status(hipError_t e) { return e == hipSuccess ? MXFP8_OK : MXFP8_ERR_HIP; }
// Entries and rows are numbered in int32; row numbers times widths are counted in 64 bits.
constexpr int64_t kMaxRows = int64_t(1) << 30, kMaxCols = int64_t(1) << 30, kMaxK = int64_t(1) << 24;
constexpr int32_t kMaxGroups = 4096, kMaxAlign = 4096, kMaxSlots = 4096;
// tokens * slots entries, each with cols values
inline bool valid_entries(int64_t tokens, int32_t slots)
{
    return tokens >= 0 && tokens <= kMaxRows && slots >= 1 && slots <= kMaxSlots && tokens * slots <= kMaxRows;
}
}  // namespace

extern "C" {

int64_t mxfp8_expert_rows(int64_t entries, int32_t groups, int32_t align)
{
    if (entries < 0 || entries > kMaxRows || groups < 0 || groups > kMaxGroups || align < 1 || align > kMaxAlign || (align & (align - 1)))
        return -1;
    const int64_t rows = (entries + (entries < groups ? entries : groups) * (align - 1)) / align * align;
    return rows <= kMaxRows ? rows : -1;
}

int64_t mxfp8_expert_sort_workspace(int64_t entries, int32_t groups)
{
    if (entries < 0 || entries > kMaxRows || groups < 0 || groups > kMaxGroups)
        return -1;
    return mxfp8::expert_sort_workspace(entries, groups);
}

mxfp8_status mxfp8_expert_sort(const void *experts, mxfp8_index experts_type, int64_t entries, int32_t groups, int32_t align,
                               int64_t rows, int32_t *positions, int32_t *sources, int32_t *group_ends, void *workspace,
                               void *hip_stream)
{
    if (experts_type != MXFP8_I32 && experts_type != MXFP8_I64)
        return MXFP8_ERR_DTYPE;
    const int64_t need = mxfp8_expert_rows(entries, groups, align);
    if (need < 0 || rows < need || rows > kMaxRows)
        return MXFP8_ERR_SHAPE;
    if (entries == 0 && rows == 0 && groups == 0)
        return MXFP8_OK;
    const bool wants_workspace = mxfp8::expert_sort_workspace(entries, groups) > 0;
    if ((entries > 0 && (!experts || !positions)) || (rows > 0 && !sources) || (groups > 0 && !group_ends) || (wants_workspace && !workspace))
        return MXFP8_ERR_NULL;
    if (!aligned(experts, experts_type == MXFP8_I64 ? 8 : 4) || !aligned(positions, 4) || !aligned(sources, 4) || !aligned(group_ends, 4) ||
        (wants_workspace && !aligned(workspace, 4)))
        return MXFP8_ERR_ALIGN;
    return status(mxfp8::launch_expert_sort(experts, experts_type == MXFP8_I64, entries, groups, align, rows, positions, sources, group_ends,
                                            static_cast<uint32_t *>(workspace), static_cast<hipStream_t>(hip_stream)));
}

mxfp8_status mxfp8_expert_quantize_ex(const void *src, mxfp8_dtype src_dtype, int64_t tokens, int64_t cols, int64_t ld_src,
                                      const int32_t *sources, int32_t slots, const float *weights, const int32_t *group_ends,
                                      int32_t groups, int64_t rows, mxfp8_axis axis, uint8_t *q_row, uint8_t *s_row,
                                      uint8_t *q_colT, uint8_t *s_colT, mxfp8_scale_layout scale_layout, void *hip_stream)
{
    if (!valid_dtype(src_dtype))
        return MXFP8_ERR_DTYPE;
    if (!valid_layout(scale_layout) || (axis != MXFP8_ROWWISE && axis != MXFP8_COLWISE && axis != MXFP8_BOTH))
        return MXFP8_ERR_MODE;
    if (!valid_entries(tokens, slots) || cols < 0 || cols > kMaxCols || cols % 32 || ld_src < cols || rows < 0 || rows > kMaxRows || rows % 32 ||
        groups < 0 || groups > kMaxGroups || (groups == 0) != (group_ends == nullptr))
        return MXFP8_ERR_SHAPE;
    if (rows == 0 || cols == 0)
        return MXFP8_OK;
    const bool want_row = axis & MXFP8_ROWWISE, want_col = axis & MXFP8_COLWISE;
    if ((tokens > 0 && !src) || !sources || (want_row && (!q_row || !s_row)) || (want_col && (!q_colT || !s_colT)))
        return MXFP8_ERR_NULL;
    if (!aligned(src, 16) || (ld_src * esize(src_dtype)) % 16 || (want_row && !aligned(q_row, 16)) || (want_col && !aligned(q_colT, 16)) ||
        !aligned(sources, 4) || !aligned(weights, 4) || !aligned(group_ends, 4))
        return MXFP8_ERR_ALIGN;
    const bool tiled = scale_layout == MXFP8_SCALES_TILED;
    if (tiled && ((want_row && !aligned(s_row, 16)) || (want_col && !aligned(s_colT, 16))))
        return MXFP8_ERR_ALIGN;
    const hipError_t e = mxfp8::launch_expert_quantize(src, src_dtype == MXFP8_BF16, tokens, cols, ld_src, sources, slots, weights, group_ends,
                                                       groups, rows, (int)axis, q_row, s_row, q_colT, s_colT, tiled,
                                                       static_cast<hipStream_t>(hip_stream));
    return e == hipErrorInvalidConfiguration ? MXFP8_ERR_SHAPE : status(e);  // more tiles than a launch can have: nothing was launched
}

mxfp8_status mxfp8_expert_combine(const void *c, mxfp8_dtype c_dtype, int64_t rows, int64_t cols, int64_t ldc,
                                  const int32_t *positions, const float *weights, int64_t tokens, int32_t slots, void *out,
                                  mxfp8_dtype out_dtype, int64_t ld_out, void *hip_stream)
{
    if (!valid_dtype(c_dtype) || !valid_dtype(out_dtype))
        return MXFP8_ERR_DTYPE;
    if (!valid_entries(tokens, slots) || rows < 0 || rows > kMaxRows || cols < 0 || cols > kMaxCols || ldc < cols || ld_out < cols)
        return MXFP8_ERR_SHAPE;
    if (tokens == 0 || cols == 0)
        return MXFP8_OK;
    if ((rows > 0 && !c) || !positions || !out)
        return MXFP8_ERR_NULL;
    if (!aligned(c, esize(c_dtype)) || !aligned(out, esize(out_dtype)) || !aligned(positions, 4) || !aligned(weights, 4))
        return MXFP8_ERR_ALIGN;
    const hipError_t e = mxfp8::launch_expert_combine(c, c_dtype == MXFP8_BF16, rows, cols, ldc, positions, weights, tokens, slots, out,
                                                      out_dtype == MXFP8_BF16, ld_out, static_cast<hipStream_t>(hip_stream));
    return e == hipErrorInvalidConfiguration ? MXFP8_ERR_SHAPE : status(e);
}

mxfp8_status mxfp8_expert_weight_grad(const void *dy, mxfp8_dtype dy_dtype, int64_t ld_dy, const void *c, mxfp8_dtype c_dtype,
                                      int64_t rows, int64_t cols, int64_t ldc, const int32_t *positions, int64_t tokens,
                                      int32_t slots, float *dweights, void *hip_stream)
{
    if (!valid_dtype(dy_dtype) || !valid_dtype(c_dtype))
        return MXFP8_ERR_DTYPE;
    if (!valid_entries(tokens, slots) || rows < 0 || rows > kMaxRows || cols < 0 || cols > kMaxCols || ldc < cols || ld_dy < cols)
        return MXFP8_ERR_SHAPE;
    if (tokens == 0)
        return MXFP8_OK;
    if ((rows > 0 && cols > 0 && !c) || (cols > 0 && !dy) || !positions || !dweights)
        return MXFP8_ERR_NULL;
    if (!aligned(c, esize(c_dtype)) || !aligned(dy, esize(dy_dtype)) || !aligned(positions, 4) || !aligned(dweights, 4))
        return MXFP8_ERR_ALIGN;
    return status(mxfp8::launch_expert_weight_grad(dy, dy_dtype == MXFP8_BF16, ld_dy, c, c_dtype == MXFP8_BF16, rows, cols, ldc, positions, tokens,
                                                   slots, dweights, static_cast<hipStream_t>(hip_stream)));
}

static mxfp8_status fp4_gemv(const void *x, int64_t tokens, int64_t ldx, const int32_t *sources, int32_t slots, const uint8_t *w_q,
                             const uint8_t *w_s, const int32_t *group_ends, int32_t groups, int64_t M, int64_t N, int64_t K, void *c,
                             mxfp8_dtype c_dtype, int64_t ldc, mxfp8_scale_layout scale_layout, void *hip_stream)
{
    const bool tiled = scale_layout == MXFP8_SCALES_TILED;
    if (!aligned(c, esize(c_dtype)) || !aligned(sources, 4) || !aligned(group_ends, 4) ||
        (K > 0 && (!aligned(x, 16) || (ldx * 2) % 16 || !aligned(w_q, 16) || (tiled && !aligned(w_s, 16)))))
        return MXFP8_ERR_ALIGN;
    const hipError_t e = mxfp8::launch_fp4_gemv(x, tokens, ldx, sources, slots, w_q, w_s, group_ends, groups, mxfp8_scale_bytes(N, K, scale_layout), M,
                                                N, K, c, c_dtype == MXFP8_BF16, ldc, tiled, static_cast<hipStream_t>(hip_stream));
    return e == hipErrorInvalidConfiguration ? MXFP8_ERR_SHAPE : status(e);
}

mxfp8_status mxfp8_fp4_gemv_ex(const void *x_bf16, int64_t ldx, const uint8_t *w_q, const uint8_t *w_s, int64_t M, int64_t N,
                               int64_t K, void *c, mxfp8_dtype c_dtype, int64_t ldc, mxfp8_scale_layout scale_layout,
                               void *hip_stream)
{
    if (!valid_dtype(c_dtype))
        return MXFP8_ERR_DTYPE;
    if (!valid_layout(scale_layout))
        return MXFP8_ERR_MODE;
    if (M < 0 || N < 0 || K < 0 || M > kMaxRows || N > kMaxCols || K > kMaxK || K % 32 || ldc < N || ldx < K)
        return MXFP8_ERR_SHAPE;
    if (M == 0 || N == 0)
        return MXFP8_OK;
    if (!c || (K > 0 && (!x_bf16 || !w_q || !w_s)))
        return MXFP8_ERR_NULL;
    return fp4_gemv(x_bf16, M, ldx, nullptr, 1, w_q, w_s, nullptr, 0, M, N, K, c, c_dtype, ldc, scale_layout, hip_stream);
}

mxfp8_status mxfp8_fp4_gemv_grouped_ex(const void *x_bf16, int64_t tokens, int64_t ldx, const int32_t *sources, int32_t slots,
                                       const uint8_t *w_q, const uint8_t *w_s, const int32_t *group_ends, int32_t groups,
                                       int64_t M, int64_t N, int64_t K, void *c, mxfp8_dtype c_dtype, int64_t ldc,
                                       mxfp8_scale_layout scale_layout, void *hip_stream)
{
    if (!valid_dtype(c_dtype))
        return MXFP8_ERR_DTYPE;
    if (!valid_layout(scale_layout))
        return MXFP8_ERR_MODE;
    if (M < 0 || N < 0 || K < 0 || M > kMaxRows || N > kMaxCols || K > kMaxK || K % 32 || ldc < N || ldx < K || groups < 0 || groups > kMaxGroups ||
        (sources ? !valid_entries(tokens, slots) : tokens < M))
        return MXFP8_ERR_SHAPE;
    if (M == 0 || N == 0 || groups == 0)
        return MXFP8_OK;
    if (!c || !group_ends || (K > 0 && ((tokens > 0 && !x_bf16) || !w_q || !w_s)))
        return MXFP8_ERR_NULL;
    return fp4_gemv(x_bf16, tokens, ldx, sources, slots, w_q, w_s, group_ends, groups, M, N, K, c, c_dtype, ldc, scale_layout, hip_stream);
}

}  // extern "C"
