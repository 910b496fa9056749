// Rows on their way to the experts and back (include/mxfp8_experts.h): the quantizer of sorted rows, the weighted sum of a
// token's rows, and the gradient of its weights. All three are bound by HBM: no row is stored between them and the products.
#include "expert_launches.h"
#include "quantize_tile.h"

#include <type_traits>

namespace mxfp8 {

// ---- quantizer of sorted rows: the tile conversion of quantize_tile.h on rows fetched through the plan ------------------------
// w * x rounded to FP32 so that it can be rounded again: to the neighbour with an odd last bit wherever it is not exact ("round to odd").
// E4M3 keeps far fewer bits, so what it rounds to, and the scale (a comparison with 1.75 * 2^n), are those of the exact product, which
// FP32's nearest value at a tie or a border is not. The rest of the product comes from a fused multiply-add; below 2^-102 it can be
// lost, and the value is then the nearest FP32 one. Infinities and NaN are the FP32 product's.
__device__ __forceinline__ uint32_t product_to_odd(float w, float x)
{
    const float p = w * x, rest = fmaf(w, x, -p);
    const uint32_t bits = __float_as_uint(p);
    const bool inexact = rest != 0.0f && (bits & 0x7F800000u) != 0x7F800000u, larger = ((__float_as_uint(rest) ^ bits) >> 31) == 0;
    return inexact && (bits & 1u) == 0 ? (larger ? bits + 1 : bits - 1) : bits;
}

// The rows of a tile, by their token (-1: zeros) and weight, in LDS. BF16 rows times an FP32 weight take the FP32 register layout.
// All loads are issued at once: rows and columns that are not there are read from the first ones and zeroed afterwards (a load each
// under a condition: BF16 [4096 tokens x 2 x 4096], both copies, with weights 49.7 us instead of 29.3).
template <bool SRC_BF16, bool WEIGHTED> struct ExpertRows {
    static constexpr bool kGiven = true;
    const uint8_t *src;
    int64_t ld_bytes;
    const int32_t *token;
    const float *weight;
    bool none;  // src has no row at all
    template <int N> __device__ __forceinline__ void load(uint4 (&x)[N], int r, int64_t c, bool active) const
    {
        const uint8_t *const from = src + (active ? c : 0) * (SRC_BF16 ? 2 : 4);
        int t[N];
        if (none) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                x[i] = make_uint4(0, 0, 0, 0);
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            t[i] = token[r + i];
            const uint8_t *p = from + max(t[i], 0) * ld_bytes;
            if constexpr (SRC_BF16 && WEIGHTED) {
                const uint2 h = *reinterpret_cast<const uint2 *>(p);
                x[i] = make_uint4(h.x, h.y, 0, 0);
            } else {
                x[i] = *reinterpret_cast<const uint4 *>(p);
            }
        }
        if constexpr (WEIGHTED) {
            // Ties and borders of the conversion end in 19 zero bits: only where a product does can it matter how it was rounded, in dense data
            // with weights that are not powers of two one tile of a wavefront in a hundred. Zeros, and BF16 values times powers of two, end in
            // them too although their products are exact. (The same tensor: never asking 29.3 us, always rounding to odd 40.8, this way 32.7;
            // with 0.1 | 1 | 10 % of the tokens zero 34.7 | 38.5 | 41.3, with weights of 1 41.4. FP32 37.4, with 1 % of the tokens zero 43.1.)
            uint32_t low = ~0u;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (SRC_BF16)
                    x[i] = make_uint4(x[i].x << 16, x[i].x & 0xFFFF0000u, x[i].y << 16, x[i].y & 0xFFFF0000u);
                const float w = weight[r + i];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    low = min(low, __float_as_uint(w * __uint_as_float(word_at(x[i], k))) & 0x7FFFFu);
            }
            if (__ballot(low == 0) != 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float w = weight[r + i];
                    x[i] = make_uint4(product_to_odd(w, __uint_as_float(x[i].x)), product_to_odd(w, __uint_as_float(x[i].y)),
                                      product_to_odd(w, __uint_as_float(x[i].z)), product_to_odd(w, __uint_as_float(x[i].w)));
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float w = weight[r + i];
                    x[i] = make_uint4(__float_as_uint(w * __uint_as_float(x[i].x)), __float_as_uint(w * __uint_as_float(x[i].y)),
                                      __float_as_uint(w * __uint_as_float(x[i].z)), __float_as_uint(w * __uint_as_float(x[i].w)));
                }
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (t[i] < 0 || !active)
                x[i] = make_uint4(0, 0, 0, 0);
    }
};

template <bool SRC_BF16, bool WEIGHTED, bool ROW, bool COL, bool TILED>
__global__ __launch_bounds__(kQuantThreads) void expert_quantize_kernel(
    const uint8_t *__restrict__ src, int64_t ld_bytes, const int32_t *__restrict__ sources, uint32_t entries, uint32_t slots,
    const float *__restrict__ weights, const int32_t *__restrict__ group_ends, int groups, int64_t rows, int64_t cols,
    uint8_t *__restrict__ q_row, uint8_t *__restrict__ s_row, uint8_t *__restrict__ q_colT, uint8_t *__restrict__ s_colT, uint32_t tiles_x)
{
    constexpr bool BF16 = SRC_BF16 && !WEIGHTED;  // register layout
    __shared__ __attribute__((aligned(16))) uint8_t lds_q[COL ? kTile * kTile : 16];
    __shared__ __attribute__((aligned(16))) uint8_t lds_rs[ROW ? kTile * 4 : 16];
    __shared__ __attribute__((aligned(16))) uint8_t lds_cs[COL ? kTile * 4 : 16];
    __shared__ int32_t token[kTile];
    __shared__ float weight[WEIGHTED ? kTile : 1];
    const QuantLds lds{lds_q, lds_rs, lds_cs, nullptr, nullptr};
    const ExpertRows<SRC_BF16, WEIGHTED> rows_of_tile{src, ld_bytes, token, weight, entries == 0};
    const int tid = threadIdx.x;
    // tiles of rows that hold a row of an expert
    const int64_t end = groups ? min(max((int64_t)group_ends[groups - 1], (int64_t)0), rows) : rows;
    const uint32_t tiles_y = (uint32_t)((end + kTile - 1) / kTile), ntiles = tiles_x * tiles_y;
    const bool walk_down = COL && cols > end;  // as in quantize.hip
    for (uint32_t tile = blockIdx.x; tile < ntiles; tile += gridDim.x) {
        const uint32_t tile_y = walk_down ? tile % tiles_y : tile / tiles_x, tile_x = walk_down ? tile / tiles_y : tile % tiles_x;
        if (tid < kTile) {
            const int64_t r = (int64_t)tile_y * kTile + tid;
            const uint32_t i = r < rows ? (uint32_t)sources[r] : ~0u;
            token[tid] = i < entries ? (int32_t)(i / slots) : -1;
            if constexpr (WEIGHTED)
                weight[tid] = i < entries ? weights[i] : 1.1f;  // of rows that become zeros: as good as never a border but for zeros of row 0
        }
        __syncthreads();
        quantize_tile<BF16, ROW, COL, TILED, 0, false>(nullptr, rows, cols, 0, q_row, s_row, q_colT, s_colT, nullptr, tile_y, tile_x, tid, lds,
                                                       &rows_of_tile);
        __syncthreads();  // between two tiles, as quantize_tile wants it (the barriers behind the next rows and within the tile would do)
    }
}

template <bool SRC_BF16, bool WEIGHTED, bool TILED>
static hipError_t launch_expert_quantize_t(const void *src, int64_t tokens, int64_t cols, int64_t ld, const int32_t *sources, int slots,
                                           const float *weights, const int32_t *group_ends, int groups, int64_t rows, int axis, uint8_t *q_row,
                                           uint8_t *s_row, uint8_t *q_colT, uint8_t *s_colT, hipStream_t stream)
{
    const int64_t tiles_x = (cols + kTile - 1) / kTile, tiles = tiles_x * ((rows + kTile - 1) / kTile);
    if (tiles > 0x7FFFFFFF)
        return hipErrorInvalidConfiguration;
    int dev = 0, cus = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e == hipSuccess)
        e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
    if (e != hipSuccess)
        return e;
    // The host knows the tiles of all rows, not how many of them belong to an expert: a resident grid walks over those that do. Four workgroups
    // a unit where a tile is large in registers (as in quantize.hip), else eight (FP32 rows times weights, row copy: 31.9 -> 27.1 us).
    const unsigned workgroups = (unsigned)min(tiles, (int64_t)max(cus, 1) * (axis == 3 ? 4 : 8));
    auto kern = axis == 1   ? expert_quantize_kernel<SRC_BF16, WEIGHTED, true, false, TILED>
                : axis == 2 ? expert_quantize_kernel<SRC_BF16, WEIGHTED, false, true, TILED>
                            : expert_quantize_kernel<SRC_BF16, WEIGHTED, true, true, TILED>;
    hipLaunchKernelGGL(kern, dim3(workgroups), dim3(kQuantThreads), 0, stream, static_cast<const uint8_t *>(src), ld * (SRC_BF16 ? 2 : 4), sources,
                       (uint32_t)(tokens * slots), (uint32_t)slots, weights, group_ends, groups, rows, cols, q_row, s_row, q_colT, s_colT,
                       (uint32_t)tiles_x);
    return hipGetLastError();
}

hipError_t launch_expert_quantize(const void *src, bool bf16, int64_t tokens, int64_t cols, int64_t ld, const int32_t *sources, int slots,
                                  const float *weights, const int32_t *group_ends, int groups, int64_t rows, int axis, uint8_t *q_row,
                                  uint8_t *s_row, uint8_t *q_colT, uint8_t *s_colT, bool tiled_scales, hipStream_t stream)
{
    auto launch = bf16 ? (weights ? (tiled_scales ? launch_expert_quantize_t<true, true, true> : launch_expert_quantize_t<true, true, false>)
                                  : (tiled_scales ? launch_expert_quantize_t<true, false, true> : launch_expert_quantize_t<true, false, false>))
                       : (weights ? (tiled_scales ? launch_expert_quantize_t<false, true, true> : launch_expert_quantize_t<false, true, false>)
                                  : (tiled_scales ? launch_expert_quantize_t<false, false, true> : launch_expert_quantize_t<false, false, false>));
    return launch(src, tokens, cols, ld, sources, slots, weights, group_ends, groups, rows, axis, q_row, s_row, q_colT, s_colT, stream);
}

// ---- sums over a token's rows --------------------------------------------------------------------------------------------------
// Up to eight consecutive values as FP32, `n` of them there. VEC: all eight always are, on 16 bytes.
struct Values8 {
    float v[8];
};
template <bool BF16, bool VEC> __device__ __forceinline__ Values8 load8(const uint8_t *p, int n)
{
    Values8 r = {};
    if constexpr (!VEC) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n)
                r.v[k] = BF16 ? __uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(p)[k] << 16) : reinterpret_cast<const float *>(p)[k];
    } else if constexpr (BF16) {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t w = word_at(a, k);
            r.v[2 * k] = __uint_as_float(w << 16);
            r.v[2 * k + 1] = __uint_as_float(w & 0xFFFF0000u);
        }
    } else {
        const uint4 a = *reinterpret_cast<const uint4 *>(p), b = *reinterpret_cast<const uint4 *>(p + 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            r.v[k] = __uint_as_float(word_at(a, k));
            r.v[4 + k] = __uint_as_float(word_at(b, k));
        }
    }
    return r;
}
template <bool BF16, bool VEC> __device__ __forceinline__ void store8(uint8_t *p, const Values8 &x, int n)
{
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const v2bf h = {(__bf16)x.v[2 * k], (__bf16)x.v[2 * k + 1]};
        w[k] = __builtin_bit_cast(uint32_t, h);
    }
    if constexpr (!VEC) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) {
                if constexpr (BF16)
                    reinterpret_cast<uint16_t *>(p)[k] = (uint16_t)(w[k / 2] >> (16 * (k & 1)));
                else
                    reinterpret_cast<float *>(p)[k] = x.v[k];
            }
    } else if constexpr (BF16) {
        stream_store(reinterpret_cast<uint4 *>(p), make_uint4(w[0], w[1], w[2], w[3]));
    } else {
        stream_store(reinterpret_cast<uint4 *>(p), make_uint4(__float_as_uint(x.v[0]), __float_as_uint(x.v[1]), __float_as_uint(x.v[2]), __float_as_uint(x.v[3])));
        stream_store(reinterpret_cast<uint4 *>(p + 16), make_uint4(__float_as_uint(x.v[4]), __float_as_uint(x.v[5]), __float_as_uint(x.v[6]), __float_as_uint(x.v[7])));
    }
}

// Whether every row of a matrix starts on 16 bytes; else its values are read and written one by one.
static bool on_16(const void *p, int64_t ld, bool bf16) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * (bf16 ? 2 : 4) % 16 == 0; }

constexpr int kRowThreads = 256, kRowWaves = kRowThreads / 64;
constexpr int kPiece = 512;  // columns of a wavefront: eight a lane
constexpr int64_t kMostWorkgroups = int64_t(1) << 22;  // work-items of a launch are numbered in 32 bits: more work is walked over

// A wavefront sums kPiece columns of one token; its rows and weights are the same for all lanes. What bounds it: HBM, the rows of c
// once. BF16 [16384 tokens x 4 x 4096] 117 us = 5.8 TB/s; a few tokens take the launch ([3 x 8 x 2048] 3.2 us in a graph, where an empty
// kernel takes 2.2; a row after the other 4.2).
template <bool C_BF16, bool OUT_BF16, bool VEC>
__global__ __launch_bounds__(kRowThreads) void expert_combine_kernel(const uint8_t *__restrict__ c, int64_t rows, int cols, int64_t ld_bytes,
                                                                     const int32_t *__restrict__ positions, const float *__restrict__ weights,
                                                                     uint32_t total, int slots, uint8_t *__restrict__ out, int64_t ld_out_bytes,
                                                                     uint32_t pieces)
{
    const int lane = threadIdx.x & 63;
    for (uint32_t id = blockIdx.x * kRowWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); id < total; id += gridDim.x * kRowWaves) {
        const uint32_t token = id / pieces;
        const int64_t col = (int64_t)(id - token * pieces) * kPiece + lane * 8;
        const int n = (int)min((int64_t)cols - col, (int64_t)8);
        if (n <= 0)
            continue;
        Values8 sum = {};
        for (int j0 = 0; j0 < slots && rows > 0; j0 += 4) {  // four rows on their way at a time; those that are not there are read as row 0
            const int64_t i = (int64_t)token * slots + j0;
            Values8 x[4];
            float w[4];
            bool there[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int32_t r = j0 + j < slots ? positions[i + j] : -1;
                there[j] = r >= 0 && r < rows;
                w[j] = weights && there[j] ? weights[i + j] : 1.0f;
                x[j] = load8<C_BF16, VEC>(c + (there[j] ? r : 0) * ld_bytes + col * (C_BF16 ? 2 : 4), n);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (there[j])
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        sum.v[k] = fmaf(w[j], x[j].v[k], sum.v[k]);
        }
        store8<OUT_BF16, VEC>(out + token * ld_out_bytes + col * (OUT_BF16 ? 2 : 4), sum, n);
    }
}

hipError_t launch_expert_combine(const void *c, bool c_bf16, int64_t rows, int64_t cols, int64_t ldc, const int32_t *positions,
                                 const float *weights, int64_t tokens, int slots, void *out, bool out_bf16, int64_t ld_out, hipStream_t stream)
{
    const int64_t pieces = (cols + kPiece - 1) / kPiece, workgroups = min((tokens * pieces + kRowWaves - 1) / kRowWaves, kMostWorkgroups);
    if (tokens * pieces > 0x7FFFFFFF)
        return hipErrorInvalidConfiguration;
    auto pick = [&](auto vec) {
        constexpr bool V = decltype(vec)::value;
        return c_bf16 ? (out_bf16 ? expert_combine_kernel<true, true, V> : expert_combine_kernel<true, false, V>)
                      : (out_bf16 ? expert_combine_kernel<false, true, V> : expert_combine_kernel<false, false, V>);
    };
    auto kern = cols % 8 == 0 && on_16(c, ldc, c_bf16) && on_16(out, ld_out, out_bf16) ? pick(std::true_type{}) : pick(std::false_type{});
    hipLaunchKernelGGL(kern, dim3((unsigned)workgroups), dim3(kRowThreads), 0, stream, static_cast<const uint8_t *>(c), rows, (int)cols,
                       ldc * (c_bf16 ? 2 : 4), positions, weights, (uint32_t)(tokens * pieces), slots, static_cast<uint8_t *>(out),
                       ld_out * (out_bf16 ? 2 : 4), (uint32_t)pieces);
    return hipGetLastError();
}

// ---- gradient of the weights ------------------------------------------------------------------------------------------------------
// A wavefront takes the dot product of one entry, a workgroup those of four entries side by side. The row of dy of a token with more slots, or
// with slots that four does not divide, is fetched by several workgroups, which lie on different XCDs with an L2 each: [1003 tokens x 6 x 2880]
// fetches dy, 11.6 MB, 1.9 times. What bounds it: HBM. BF16 [8192 x 2 x 5632] 46.9 us = 5.9 TB/s launched one after the other and 49.2 in
// a captured graph, [4096 x 8 x 2048] 29.4 there (a piece after the other 36.8), one token's 8 x 4096 3.2 (5.2).
template <bool DY_BF16, bool C_BF16, bool VEC>
__global__ __launch_bounds__(kRowThreads) void expert_weight_grad_kernel(const uint8_t *__restrict__ dy, int64_t ld_dy_bytes, const uint8_t *__restrict__ c,
                                                                         int64_t rows, int cols, int64_t ld_bytes,
                                                                         const int32_t *__restrict__ positions, uint32_t entries, uint32_t slots,
                                                                         float *__restrict__ dw)
{
    const int lane = threadIdx.x & 63;
    for (uint32_t i = blockIdx.x * kRowWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); i < entries; i += gridDim.x * kRowWaves) {
        const int32_t r = positions[i];
        Values8 part = {};
        if (r >= 0 && r < rows) {
            const uint8_t *a = dy + (int64_t)(i / slots) * ld_dy_bytes, *b = c + r * ld_bytes;
            int64_t col = lane * 8;
            for (; col + 3 * kPiece + 8 <= cols; col += 4 * kPiece) {  // four pieces on their way at a time
                Values8 x[4], y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[j] = load8<DY_BF16, VEC>(a + (col + j * kPiece) * (DY_BF16 ? 2 : 4), 8);
                    y[j] = load8<C_BF16, VEC>(b + (col + j * kPiece) * (C_BF16 ? 2 : 4), 8);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        part.v[k] = fmaf(x[j].v[k], y[j].v[k], part.v[k]);
            }
            for (; col < cols; col += kPiece) {
                const int n = (int)min((int64_t)cols - col, (int64_t)8);
                const Values8 x = load8<DY_BF16, VEC>(a + col * (DY_BF16 ? 2 : 4), n), y = load8<C_BF16, VEC>(b + col * (C_BF16 ? 2 : 4), n);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    part.v[k] = fmaf(x.v[k], y.v[k], part.v[k]);
            }
        }
        float sum = ((part.v[0] + part.v[1]) + (part.v[2] + part.v[3])) + ((part.v[4] + part.v[5]) + (part.v[6] + part.v[7]));
        for (int d = 32; d >= 1; d /= 2)
            sum += __uint_as_float((uint32_t)__shfl_xor((int)__float_as_uint(sum), d, 64));
        if (lane == 0)
            dw[i] = sum;
    }
}

hipError_t launch_expert_weight_grad(const void *dy, bool dy_bf16, int64_t ld_dy, const void *c, bool c_bf16, int64_t rows, int64_t cols,
                                     int64_t ldc, const int32_t *positions, int64_t tokens, int slots, float *dw, hipStream_t stream)
{
    const int64_t entries = tokens * slots, workgroups = min((entries + kRowWaves - 1) / kRowWaves, kMostWorkgroups);
    auto pick = [&](auto vec) {
        constexpr bool V = decltype(vec)::value;
        return dy_bf16 ? (c_bf16 ? expert_weight_grad_kernel<true, true, V> : expert_weight_grad_kernel<true, false, V>)
                       : (c_bf16 ? expert_weight_grad_kernel<false, true, V> : expert_weight_grad_kernel<false, false, V>);
    };
    auto kern = cols % 8 == 0 && on_16(c, ldc, c_bf16) && on_16(dy, ld_dy, dy_bf16) ? pick(std::true_type{}) : pick(std::false_type{});
    hipLaunchKernelGGL(kern, dim3((unsigned)workgroups), dim3(kRowThreads), 0, stream, static_cast<const uint8_t *>(dy), ld_dy * (dy_bf16 ? 2 : 4),
                       static_cast<const uint8_t *>(c), rows, (int)cols, ldc * (c_bf16 ? 2 : 4), positions, (uint32_t)entries, (uint32_t)slots, dw);
    return hipGetLastError();
}

}  // namespace mxfp8
