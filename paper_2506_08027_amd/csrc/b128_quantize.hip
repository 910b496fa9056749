// Quantizer to E4M3 with an FP32 scale for each block of 128 (include/mxfp8_b128.h): X = amax / 448, Q_i = RNE(V_i / X).
//
// A workgroup converts a tile of 128 x 128: it is read once, 8 x 8 values a thread (8 consecutive columns of 8 consecutive rows),
// which stay in registers for both copies. A row's 16 threads lie in one row of 16 lanes, so its largest magnitude takes four DPP
// steps; a column's 16 threads lie in four wavefronts and meet in LDS. The transposed copy's bytes go through LDS, eight rows of a
// column a store, so that the rows of both copies leave as whole 128-byte lines.
//   The quotient V / X is the FP32 one, correctly rounded: t = V r with r = RN(1 / X), corrected by its exact remainder,
// t - (t X - V) r. A plain V r is often one unit off, and where V / X lies on a border between two codes (3 / 64 of the block's largest
// value does) that unit decides between them. It is exact as long as no remainder is rounded away: blocks with a largest magnitude below
// 2^-60 (but not 0), where one could be, and blocks with infinities or NaN take the division instead, in code of its own.
//   What bounds it: HBM, with one read and two write streams. BF16 [8192 x 4096], both copies 28 us (4.8 TB/s), row copy 19.8 (5.1); FP32
// [14336 x 4096] in tiles, both copies 66.7 (5.3); FP32 [1999 x 5632], both copies 19.2: there the values take 64 registers and their
// conversion 168 in all, three workgroups of four wavefronts to a unit: 704 tiles are one round, whose reads, conversions and writes overlap little.
#include "b128_launches.h"
#include "mxfp8_device.h"

#include <float.h>
#include <type_traits>

namespace mxfp8 {

constexpr int kWide = 128;           // values of a block
// Place of rows 8 s .. 8 s + 7 of column c of the tile in LDS: XORed, so that lanes that write or read the same rows of columns 8 apart
// hit different banks.
__device__ __forceinline__ int staged_place(int c, int s) { return c * kWide + ((s ^ (c >> 3)) & 15) * 8; }

// 16 lanes of a row
__device__ __forceinline__ uint32_t max_of_16(uint32_t v)
{
    v = umax(v, dpp_xor1(v));
    v = umax(v, dpp_xor2(v));
    v = umax(v, dpp_half_mirror(v));
    return umax(v, dpp_mirror(v));
}

struct WideScale {
    float x, inverse;  // inverse 0: not by the plain way (infinities, NaN, remainders below the FP32 range)
};
__device__ __forceinline__ WideScale wide_scale(uint32_t amax_bits)
{
    const float amax = fminf(__uint_as_float(amax_bits), FLT_MAX);
    float x = amax / 448.0f;
    x = x < 0x1p-126f ? 0x1p-126f : x;
    return {amax_bits > 0x7F800000u ? __uint_as_float(0x7FC00000u) : x, amax_bits == 0 || (amax_bits >= 0x21800000u && amax_bits < 0x7F800000u) ? 1.0f / x : 0.0f};  // 2^-60
}
__device__ __forceinline__ float wide_quotient(float v, const WideScale &s)
{
    const float t = v * s.inverse;
    return __builtin_fmaf(-__builtin_fmaf(t, s.x, -v), s.inverse, t);  // (these signs keep that of a zero)
}
// a, b of one block as codes in a half of `old`
__device__ __forceinline__ uint32_t wide_codes(uint32_t old, float a, float b, const WideScale &s, bool hi)
{
    return cvt2_f32(old, wide_quotient(a, s), wide_quotient(b, s), 1.0f, hi);
}
// one code of any block
__device__ __forceinline__ uint32_t wide_code_any(float v, const WideScale &s)
{
    if (s.x != s.x)
        return 0x7Fu;
    return cvt2_f32(0, fmaxf(fminf(v, FLT_MAX), -FLT_MAX) / s.x, 0.0f, 1.0f, false) & 0xFFu;
}
// value of lane I of the 16 lanes of a row
template <int I> __device__ __forceinline__ float of_lane(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x150 + I, 0xF, 0xF, true));
}

// AXIS: mxfp8_axis. VEC: the source and its rows are 16-byte aligned.
template <bool BF16, int AXIS, bool TILES, bool VEC>
__global__ __launch_bounds__(256) void b128_quantize_kernel(const uint8_t *__restrict__ src, int rows, int cols, int64_t ld, uint32_t tiles_c,
                                                            uint8_t *__restrict__ q_row, int64_t ld_row, float *__restrict__ s_row,
                                                            uint8_t *__restrict__ q_colT, int64_t ld_colT, float *__restrict__ s_colT)
{
    constexpr bool ROW = AXIS & 1, COL = AXIS & 2;
    constexpr int ESZ = BF16 ? 2 : 4;
    __shared__ uint4 staged[COL ? kWide * kWide / 16 : 1];
    __shared__ uint32_t maxima[4][kWide];
    typedef float ScalePair __attribute__((ext_vector_type(2)));
    __shared__ ScalePair scales[kWide];
    __shared__ uint32_t other_ways[2];  // whether a column of the tile's halves does not go the plain way
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int piece = tid & 15, group = tid >> 4;  // columns 8 piece .., rows 8 group .. of the tile
    const int tile_r = (int)(blockIdx.x / tiles_c), tile_c = (int)(blockIdx.x % tiles_c);
    const int r0 = tile_r * kWide + group * 8, c0 = tile_c * kWide + piece * 8;
    const int rows16 = (rows + 15) & ~15, cols16 = (cols + 15) & ~15;

    uint32_t w[8][BF16 ? 4 : 8];  // values as they were read
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint8_t *const at = src + ((int64_t)(r0 + i) * ld + c0) * ESZ;
#pragma unroll
        for (int j = 0; j < (BF16 ? 4 : 8); ++j)
            w[i][j] = 0;
        if (r0 + i < rows && c0 < cols) {
            if (VEC && c0 + 8 <= cols) {
                uint4 a = stream_load(reinterpret_cast<const uint4 *>(at));
                w[i][0] = a.x, w[i][1] = a.y, w[i][2] = a.z, w[i][3] = a.w;
                if constexpr (!BF16) {
                    a = stream_load(reinterpret_cast<const uint4 *>(at) + 1);
                    w[i][4] = a.x, w[i][5] = a.y, w[i][6] = a.z, w[i][7] = a.w;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c0 + j < cols) {
                        if constexpr (BF16)
                            w[i][j / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(at)[j] << (16 * (j & 1));
                        else
                            w[i][j] = reinterpret_cast<const uint32_t *>(at)[j];
                    }
            }
        }
    }
    auto value = [&](int i, int j) __attribute__((always_inline)) {
        return __uint_as_float(BF16 ? (j & 1 ? w[i][j / 2] & 0xFFFF0000u : w[i][j / 2] << 16) : w[i][BF16 ? 0 : j]);
    };
    // magnitudes of word j, as they are compared: two BF16 ones at once
    auto magnitude = [&](int i, int j) __attribute__((always_inline)) { return w[i][j] & (BF16 ? 0x7FFF7FFFu : 0x7FFFFFFFu); };
    auto larger = [](uint32_t a, uint32_t b) __attribute__((always_inline)) { return BF16 ? pk_max_u16(a, b) : umax(a, b); };
    constexpr int WORDS = BF16 ? 4 : 8;

    // ---- eight codes of a line of values. ANY: some block of the wavefront may not go the plain way; zeros from `given` on
    auto line = [](const float (&x)[8], const WideScale &s, int given, auto any) __attribute__((always_inline)) {
        if (!decltype(any)::value || s.inverse != 0.0f)
            return make_uint2(wide_codes(wide_codes(0, x[0], x[1], s, false), x[2], x[3], s, true),
                              wide_codes(wide_codes(0, x[4], x[5], s, false), x[6], x[7], s, true));
        uint32_t lo = 0, hi = 0;
        for (int j = 0; j < 4; ++j) {
            lo |= (j < given ? wide_code_any(x[j], s) : 0u) << (8 * j);
            hi |= (4 + j < given ? wide_code_any(x[4 + j], s) : 0u) << (8 * j);
        }
        return make_uint2(lo, hi);
    };
    auto row_codes = [&](int i, const WideScale &s, auto any) __attribute__((always_inline)) {
        const float x[8] = {value(i, 0), value(i, 1), value(i, 2), value(i, 3), value(i, 4), value(i, 5), value(i, 6), value(i, 7)};
        return line(x, s, cols - c0, any);
    };
    auto store_row = [&](int i, uint2 q) __attribute__((always_inline)) {
        if (r0 + i < rows && c0 < cols16)
            stream_store(reinterpret_cast<uint2 *>(q_row + (int64_t)(r0 + i) * ld_row + c0), q);
    };
    uint8_t *const area = reinterpret_cast<uint8_t *>(staged);
    auto row_max = [&](int i) __attribute__((always_inline)) {
        uint32_t m = magnitude(i, 0);
#pragma unroll
        for (int j = 1; j < WORDS; ++j)
            m = larger(m, magnitude(i, j));
        return BF16 ? umax(m << 16, m & 0xFFFF0000u) : m;
    };

    if constexpr (TILES) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            m = umax(m, row_max(i));
        m = max_of_16(m);
        m = umax(m, (uint32_t)__shfl_xor((int)m, 16, 64));
        m = umax(m, (uint32_t)__shfl_xor((int)m, 32, 64));
        if (lane == 0)
            maxima[wave][0] = m;
        __syncthreads();
        const WideScale s = wide_scale(umax(umax(maxima[0][0], maxima[1][0]), umax(maxima[2][0], maxima[3][0])));
        uint2 q[8];
        if (s.inverse != 0.0f) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                q[i] = row_codes(i, s, std::false_type{});
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                q[i] = row_codes(i, s, std::true_type{});
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (r0 + i >= rows)
                q[i] = make_uint2(0, 0);
            if constexpr (ROW)
                store_row(i, q[i]);
        }
        if constexpr (COL)  // the same codes: 4 x 4 of them at a time, turned
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t c[2][4];  // of rows 0 .. 3 and 4 .. 7
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t a = half ? q[4 * k].y : q[4 * k].x, b = half ? q[4 * k + 1].y : q[4 * k + 1].x, d = half ? q[4 * k + 2].y : q[4 * k + 2].x,
                                   e = half ? q[4 * k + 3].y : q[4 * k + 3].x;
                    const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400), ab2 = __builtin_amdgcn_perm(b, a, 0x07030602),
                                   de0 = __builtin_amdgcn_perm(e, d, 0x05010400), de2 = __builtin_amdgcn_perm(e, d, 0x07030602);
                    c[k][0] = __builtin_amdgcn_perm(de0, ab0, 0x05040100), c[k][1] = __builtin_amdgcn_perm(de0, ab0, 0x07060302);
                    c[k][2] = __builtin_amdgcn_perm(de2, ab2, 0x05040100), c[k][3] = __builtin_amdgcn_perm(de2, ab2, 0x07060302);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<uint2 *>(area + staged_place(piece * 8 + half * 4 + j, group)) = make_uint2(c[0][j], c[1][j]);
            }
        if (tid == 0) {
            if constexpr (ROW)
                s_row[blockIdx.x] = s.x;
            if constexpr (COL)
                s_colT[(int64_t)tile_c * (gridDim.x / tiles_c) + tile_r] = s.x;
        }
    } else {
        uint32_t row_maxima[8];  // (here, so that the magnitudes are not kept for it)
        if constexpr (ROW)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                row_maxima[i] = row_max(i);
        if constexpr (COL) {
            uint32_t col_max[8];
#pragma unroll
            for (int j = 0; j < WORDS; ++j) {
                uint32_t m = magnitude(0, j);
#pragma unroll
                for (int i = 1; i < 8; ++i)
                    m = larger(m, magnitude(i, j));
                m = larger(m, (uint32_t)__shfl_xor((int)m, 16, 64));
                m = larger(m, (uint32_t)__shfl_xor((int)m, 32, 64));
                if constexpr (BF16)
                    col_max[2 * j] = m << 16, col_max[2 * j + 1] = m & 0xFFFF0000u;
                else
                    col_max[j] = m;
            }
            if (lane < 16) {
                *reinterpret_cast<uint4 *>(&maxima[wave][piece * 8]) = make_uint4(col_max[0], col_max[1], col_max[2], col_max[3]);
                *reinterpret_cast<uint4 *>(&maxima[wave][piece * 8 + 4]) = make_uint4(col_max[4], col_max[5], col_max[6], col_max[7]);
            }
            __syncthreads();
            if (tid < kWide) {  // a thread for each column makes its scale
                const WideScale s = wide_scale(umax(umax(maxima[0][tid], maxima[1][tid]), umax(maxima[2][tid], maxima[3][tid])));
                scales[tid] = ScalePair{s.x, s.inverse};
                const uint64_t other = __ballot(s.inverse == 0.0f);
                if (lane == 0)
                    other_ways[wave] = other != 0;
                if (tile_c * kWide + tid < cols)
                    s_colT[(int64_t)tile_r * cols + tile_c * kWide + tid] = s.x;
            }
        }
        __builtin_amdgcn_sched_barrier(0);  // (rows and columns at once, or all rows, would take twice the registers)
        if constexpr (ROW) {  // lane i of a row's sixteen makes the scale of its row i
            uint32_t mine = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t m = max_of_16(row_maxima[i]);
                mine = (lane & 7) == i ? m : mine;
            }
            const WideScale s = wide_scale(mine);
            if (piece < 8 && r0 + piece < rows)
                s_row[(int64_t)tile_c * rows + r0 + piece] = s.x;
            auto convert = [&](auto any) __attribute__((always_inline)) {
                auto one = [&](int i, const WideScale &of_row) __attribute__((always_inline)) {
                    store_row(i, row_codes(i, of_row, any));
                    __builtin_amdgcn_sched_barrier(0);
                };
                one(0, {of_lane<0>(s.x), of_lane<0>(s.inverse)});
                one(1, {of_lane<1>(s.x), of_lane<1>(s.inverse)});
                one(2, {of_lane<2>(s.x), of_lane<2>(s.inverse)});
                one(3, {of_lane<3>(s.x), of_lane<3>(s.inverse)});
                one(4, {of_lane<4>(s.x), of_lane<4>(s.inverse)});
                one(5, {of_lane<5>(s.x), of_lane<5>(s.inverse)});
                one(6, {of_lane<6>(s.x), of_lane<6>(s.inverse)});
                one(7, {of_lane<7>(s.x), of_lane<7>(s.inverse)});
            };
            if (__ballot(s.inverse == 0.0f))
                convert(std::true_type{});
            else
                convert(std::false_type{});
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (COL) {
            __syncthreads();
            auto convert = [&](auto any) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x[8] = {value(0, j), value(1, j), value(2, j), value(3, j), value(4, j), value(5, j), value(6, j), value(7, j)};
                    const ScalePair s = scales[piece * 8 + j];
                    *reinterpret_cast<uint2 *>(area + staged_place(piece * 8 + j, group)) = line(x, {s[0], s[1]}, rows - r0, any);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            if (other_ways[0] | other_ways[1])
                convert(std::true_type{});
            else
                convert(std::false_type{});
        }
    }
    if constexpr (COL) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int c = t * 32 + (tid >> 3), r = (tid & 7) * 16;
            if (tile_c * kWide + c < cols && tile_r * kWide + r < rows16) {
                const uint2 a = *reinterpret_cast<const uint2 *>(area + staged_place(c, r / 8)), b = *reinterpret_cast<const uint2 *>(area + staged_place(c, r / 8 + 1));
                stream_store(reinterpret_cast<uint4 *>(q_colT + (int64_t)(tile_c * kWide + c) * ld_colT + tile_r * kWide + r), make_uint4(a.x, a.y, b.x, b.y));
            }
        }
    }
}

hipError_t launch_b128_quantize(const void *src, bool bf16, int64_t rows, int64_t cols, int64_t ld, int axis, bool tiles, uint8_t *q_row, int64_t ld_row,
                                float *s_row, uint8_t *q_colT, int64_t ld_colT, float *s_colT, hipStream_t stream)
{
    const int64_t tiles_r = (rows + kWide - 1) / kWide, tiles_c = (cols + kWide - 1) / kWide;
    const bool vec = reinterpret_cast<uintptr_t>(src) % 16 == 0 && ld * (bf16 ? 2 : 4) % 16 == 0;
    auto launch = [&](auto is_bf16, auto ax, auto in_tiles, auto aligned) {
        constexpr bool B = decltype(is_bf16)::value, T = decltype(in_tiles)::value, V = decltype(aligned)::value;
        constexpr int A = decltype(ax)::value;
        auto kern = b128_quantize_kernel<B, A, T, V>;
        hipLaunchKernelGGL(kern, dim3((unsigned)(tiles_r * tiles_c)), dim3(256), 0, stream, static_cast<const uint8_t *>(src), (int)rows, (int)cols, ld,
                           (uint32_t)tiles_c, q_row, ld_row, s_row, q_colT, ld_colT, s_colT);
        return hipGetLastError();
    };
    auto with_vec = [&](auto b, auto a, auto t) { return vec ? launch(b, a, t, std::true_type{}) : launch(b, a, t, std::false_type{}); };
    auto with_tiles = [&](auto b, auto a) { return tiles ? with_vec(b, a, std::true_type{}) : with_vec(b, a, std::false_type{}); };
    auto with_axis = [&](auto b) {
        return axis == 1   ? with_tiles(b, std::integral_constant<int, 1>{})
               : axis == 2 ? with_tiles(b, std::integral_constant<int, 2>{})
                           : with_tiles(b, std::integral_constant<int, 3>{});
    };
    return bf16 ? with_axis(std::true_type{}) : with_axis(std::false_type{});
}

}  // namespace mxfp8
