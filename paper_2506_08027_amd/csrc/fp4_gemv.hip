// Products of a few rows of BF16 activations with MXFP4 weights (include/mxfp8_experts.h): C[m, n] = sum_k x[m, k] W[n, k].
//
// Every weight is read once for up to 16 rows of x, so HBM is the bound as long as the matrix and LDS work hide behind it. A workgroup
// has 16 rows of W and all of K, its wavefronts take turns at K and their sums are joined in LDS. The 4-bit codes
// are widened to BF16, scale included, by v_cvt_scalef32_pk_bf16_fp4 (exact where BF16 holds the value), and multiplied on
// v_mfma_f32_16x16x32_bf16. That instruction takes 8 consecutive k a lane, but any order of k will do that x and W share: lane 16g + r
// loads the 16 bytes of block 4u + g of weight row r, a whole scale block, and instruction i of four takes their elements
// 8i .. 8i + 7; the lane's scale byte applies to all of them.
#include "expert_launches.h"
#include "gemm_device.h"

namespace mxfp8 {

constexpr int kUnit = 4;            // scale blocks of a unit: 128 k, 64 bytes of a weight row
constexpr int kGemvWaves = 8, kGemvThreads = 64 * kGemvWaves;
constexpr int kXLds = 64 * 1024;    // LDS for the activations

// two bytes of E2M1 codes -> ... eight codes of a word as BF16, times the scale
__device__ __forceinline__ v8bf fp4_word_bf16(uint32_t w, float scale)
{
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

struct GemvRows {
    const int32_t *sources;  // nullptr: row r of C takes row r of x
    uint32_t entries, slots;
    const int32_t *ends;     // nullptr: one weight matrix for all rows
    int groups;
    int64_t wq_group_bytes, ws_group_bytes;
};

// Rows [first, first + count) of C with the weights of one expert: piece `u` of all experts' rows cut into pieces of R.
struct GemvPiece {
    int expert, first, count;
};
template <int R> __device__ __forceinline__ GemvPiece grouped_piece(const int32_t *__restrict__ ends, int groups, int M, int u, int lane)
{
    int before = 0;  // pieces of the experts before e0
    for (int e0 = 0; e0 < groups; e0 += 64) {
        const int e = e0 + lane;
        const int end = e < groups ? min(max(ends[e], 0), M) : 0, begin = e < groups && e > 0 ? min(max(ends[e - 1], 0), M) : 0;
        const int rows = max(end - begin, 0), n = (rows + R - 1) / R;
        int upto = n;
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl(upto, lane >= d ? lane - d : lane, 64);
            upto += lane >= d ? o : 0;
        }
        const uint64_t past = __ballot(before + upto > u);
        if (past) {
            const int l = __builtin_ctzll(past);
            const int k = u - before - (__shfl(upto, l, 64) - __shfl(n, l, 64));
            return {e0 + l, __shfl(begin, l, 64) + k * R, min(__shfl(rows, l, 64) - k * R, R)};
        }
        before += __shfl(upto, 63, 64);
    }
    return {0, 0, 0};
}

// MT tiles of 16 rows of x. x in LDS: [unit][row][16 pieces of 16 bytes], piece 4g + i at place (4g + i) ^ (row & 15), so that the
// sixteen rows that a fragment read touches lie in different banks.
template <int MT, bool TILED, bool GROUPED>
__global__ __launch_bounds__(kGemvThreads) void fp4_gemv_kernel(const uint8_t *__restrict__ x, int64_t ldx_bytes, GemvRows map,
                                                                const uint8_t *__restrict__ w_q, const uint8_t *__restrict__ w_s, int M, int N, int nb,
                                                                uint32_t tiles_n, uint8_t *__restrict__ c, bool c_bf16, int64_t ldc, bool c_vector)
{
    MXFP8_DYNAMIC_LDS(lds);
    __shared__ int64_t x_row[MT * 16];  // byte offset of a row of x, -1: zeros
    constexpr int R = MT * 16;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g = lane >> 4;
    const uint32_t tile = blockIdx.x % tiles_n, u_piece = blockIdx.x / tiles_n;
    GemvPiece p;
    if constexpr (GROUPED)
        p = grouped_piece<R>(map.ends, map.groups, M, (int)u_piece, lane);
    else
        p = {0, (int)u_piece * R, min(M - (int)u_piece * R, R)};
    if (p.count <= 0)
        return;
    if (tid < p.count) {
        const int row = p.first + tid;
        int64_t at = row;
        if (GROUPED && map.sources) {
            const uint32_t i = (uint32_t)map.sources[row];
            at = i < map.entries ? (int64_t)(i / map.slots) : -1;
        }
        x_row[tid] = at < 0 ? -1 : at * ldx_bytes;
    }
    const int units = (nb + kUnit - 1) / kUnit;
    // rows of x in LDS: a power of two; units that fit beside each other
    int held = 1;
    while (held < p.count)
        held *= 2;
    const int held_log = 31 - __builtin_clz((unsigned)held), chunk = kXLds / 256 >> held_log;

    const int n0 = (int)tile * 16, wrow = min(n0 + r, N - 1);
    const int64_t k_bytes = (int64_t)nb * 16;
    const uint8_t *wq = w_q + p.expert * (GROUPED ? map.wq_group_bytes : 0) + wrow * k_bytes;
    const uint8_t *ws = w_s + p.expert * (GROUPED ? map.ws_group_bytes : 0);
    ws += TILED ? ((int64_t)(wrow >> 6) * ((nb + 3) / 4) * 64 + (wrow & 63)) * 4 : (int64_t)wrow * nb;

    v4f acc[MT] = {};
    for (int c0 = 0; c0 < units; c0 += chunk) {
        const int here = min(chunk, units - c0);
        __syncthreads();  // x_row is there; the last chunk has been read
        const int pieces = here * 16;
        for (int m = 0; m < p.count; ++m) {
            const int64_t row = x_row[m];
            for (int q = tid; q < pieces; q += kGemvThreads) {
                const int unit = q >> 4, piece = q & 15;
                uint4 v = make_uint4(0, 0, 0, 0);
                if (row >= 0 && (c0 + unit) * kUnit + (piece >> 2) < nb)
                    v = *reinterpret_cast<const uint4 *>(x + row + (int64_t)c0 * 256 + q * 16);
                *reinterpret_cast<uint4 *>(lds + ((unit * held + m) * 16 + (piece ^ (m & 15))) * 16) = v;
            }
        }
        __syncthreads();
        for (int u = wave; u < here; u += kGemvWaves) {
            const int b = (c0 + u) * kUnit + g;  // this lane's block; blocks past the end are zeros
            const bool there = b < nb;
            uint4 w = make_uint4(0, 0, 0, 0);
            uint32_t sb = 127;
            if (there) {
                w = *reinterpret_cast<const uint4 *>(wq + (int64_t)b * 16);
                sb = TILED ? ws[(int64_t)(b >> 2) * 256 + (b & 3)] : ws[b];
            }
            const float scale = scale_operand(sb);
            const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const v8bf a = fp4_word_bf16(words[i], scale);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const int m = min(t * 16 + r, held - 1);
                    const v4i f = *reinterpret_cast<const v4i *>(lds + ((u * held + m) * 16 + ((4 * g + i) ^ (m & 15))) * 16);
                    acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(v8bf, f), acc[t], 0, 0, 0);
                }
            }
        }
    }

    // ---- the wavefronts' sums, in their order
    __syncthreads();
    v4f *const sums = reinterpret_cast<v4f *>(lds);
#pragma unroll
    for (int t = 0; t < MT; ++t)
        sums[(wave * MT + t) * 64 + lane] = acc[t];
    __syncthreads();
    if (wave >= MT)
        return;
    v4f sum = sums[wave * 64 + lane];
    for (int w = 1; w < kGemvWaves; ++w)
        sum += sums[(w * MT + wave) * 64 + lane];
    const int m = wave * 16 + r, n = n0 + 4 * g;
    if (m >= p.count || n >= N)
        return;
    uint8_t *const to = c + ((p.first + m) * ldc + n) * (c_bf16 ? 2 : 4);
    if (c_bf16) {
        const v2bf a = {(__bf16)sum[0], (__bf16)sum[1]}, b = {(__bf16)sum[2], (__bf16)sum[3]};
        const uint2 h = make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
        if (c_vector && n + 4 <= N) {
            *reinterpret_cast<uint2 *>(to) = h;
        } else {
            for (int v = 0; v < 4 && n + v < N; ++v)
                reinterpret_cast<uint16_t *>(to)[v] = (uint16_t)((v < 2 ? h.x : h.y) >> (16 * (v & 1)));
        }
    } else {
        if (c_vector && n + 4 <= N) {
            *reinterpret_cast<v4f *>(to) = sum;
        } else {
            for (int v = 0; v < 4 && n + v < N; ++v)
                reinterpret_cast<float *>(to)[v] = sum[v];
        }
    }
}

hipError_t launch_fp4_gemv(const void *x, int64_t tokens, int64_t ldx, const int32_t *sources, int slots, const uint8_t *w_q, const uint8_t *w_s,
                           const int32_t *group_ends, int groups, int64_t ws_group_bytes, int64_t M, int64_t N, int64_t K, void *c, bool c_bf16,
                           int64_t ldc, bool tiled_scales, hipStream_t stream)
{
    const bool grouped = group_ends != nullptr;
    const int64_t rows = grouped ? (M + groups - 1) / groups : M;  // of a matrix, in the mean
    const int mt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4, R = 16 * mt;
    // an expert's rows take at most one piece more than they fill
    const int64_t some = grouped ? min((int64_t)groups, M) : 0, pieces = grouped ? some + (M - some) / R : (M + R - 1) / R;
    const int64_t tiles_n = (N + 15) / 16, workgroups = tiles_n * pieces;
    if (workgroups > 0x7FFFFFFF)
        return hipErrorInvalidConfiguration;
    const GemvRows map = {sources, (uint32_t)(tokens * slots), (uint32_t)slots, group_ends, groups, N * (K / 2), ws_group_bytes};
    const int64_t es = c_bf16 ? 2 : 4;
    const bool vector = reinterpret_cast<uintptr_t>(c) % 16 == 0 && (ldc * es) % 16 == 0;
    auto pick = [&](auto one, auto two, auto four) { return mt == 1 ? one : mt == 2 ? two : four; };
    auto kern = grouped ? (tiled_scales ? pick(fp4_gemv_kernel<1, true, true>, fp4_gemv_kernel<2, true, true>, fp4_gemv_kernel<4, true, true>)
                                        : pick(fp4_gemv_kernel<1, false, true>, fp4_gemv_kernel<2, false, true>, fp4_gemv_kernel<4, false, true>))
                        : (tiled_scales ? pick(fp4_gemv_kernel<1, true, false>, fp4_gemv_kernel<2, true, false>, fp4_gemv_kernel<4, true, false>)
                                        : pick(fp4_gemv_kernel<1, false, false>, fp4_gemv_kernel<2, false, false>, fp4_gemv_kernel<4, false, false>));
    hipLaunchKernelGGL(kern, dim3((unsigned)workgroups), dim3(kGemvThreads), kXLds, stream, static_cast<const uint8_t *>(x), ldx * 2, map, w_q, w_s,
                       (int)M, (int)N, (int)(K / kBlock), (uint32_t)tiles_n, static_cast<uint8_t *>(c), c_bf16, ldc, vector);
    return hipGetLastError();
}

}  // namespace mxfp8
