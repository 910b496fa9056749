// Products of a few rows of BF16 activations with MXFP4 weights (include/mxfp8_experts.h): C[m, n] = sum_k x[m, k] W[n, k].
//
// Every weight is read once for up to 32 rows of x, so HBM is the bound as long as all else hides behind it. A wavefront takes 16 rows of
// W and a contiguous part of K, in units of 128 k: the 4-bit codes are widened to BF16, scale included, by
// v_cvt_scalef32_pk_bf16_fp4 (exact where BF16 holds the value) and multiplied on v_mfma_f32_16x16x32_bf16, W as its first operand. Where a
// workgroup's wavefronts share rows of W, their sums are joined in LDS in a fixed order; until then no wavefront waits for another.
//   Layout. The instruction takes 8 consecutive k a lane, but any order of k will do that x and W share: lane 16g + r has block g of a unit of
//   weight row r, a whole scale block, and instruction i of four multiplies its elements 8i .. 8i + 7. Loaded in that order, neighbouring lanes
//   would read different rows and a load would take four times its time in the address unit (measured: x and W read in place, [12 x 4096 x
//   14336] 17.4 us). So four neighbouring lanes load 64 bytes of a row of W and 16 lanes 256 bytes of a row of x, and each
//   wavefront reorders them through an LDS area of its own. Rows that are not there are read from one that is, and their column of the
//   result is dropped: a load under a condition would have to be waited for before the loads behind it.
//   Measured in a captured graph, where an empty kernel takes 2.2 us: [1 x 4096 x 4096] 5.0 us, [1 x 4096 x 14336] 10.4 and [1 x 28672 x 4096]
//   15.6 (9, 31 and 62 MB of weights: what comes on top of the first goes at 4.1 TB/s where K is long, at 5.0 where there are many rows
//   of W), 48 tokens x 4 of 64 experts [5632 x 2048] 74 (45 to 53 of the experts are chosen, 280 to 330 MB: 4.2 TB/s). With more rows
//   the copies of x that each workgroup fetches from L2 take over: [12 x 4096 x 14336] 14.2 us (88 MB of x beside 31 of W),
//   [64 x 28672 x 4096] 44.
#include "expert_launches.h"
#include "gemm_device.h"

#include <type_traits>

namespace mxfp8 {

constexpr int kUnit = 4;  // scale blocks of a unit: 128 k, 64 bytes of a weight row, 256 bytes of a row of x
constexpr int kGemvWaves = 8, kGemvThreads = 64 * kGemvWaves;
constexpr int64_t kMostGemvWorkgroups = (int64_t(1) << 23) - 1;  // work-items of a launch are numbered in 32 bits

// the eight codes of a word as BF16, times the scale
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
    int before = 0, last_end = 0;  // pieces of the experts before e0, and the end of the last of them
    for (int e0 = 0; e0 < groups; e0 += 64) {
        const int e = e0 + lane;
        const int end = e < groups ? min(max(ends[e], 0), M) : 0;
        const int prev = __shfl(end, max(lane - 1, 0), 64), begin = lane == 0 ? last_end : prev;
        const int rows = e < groups ? max(end - begin, 0) : 0, n = (rows + R - 1) / R;
        int upto = n;  // inclusive sum: over the rows of 16 lanes, then over those
        upto += (int)__builtin_amdgcn_update_dpp(0, upto, 0x111, 0xF, 0xF, true);
        upto += (int)__builtin_amdgcn_update_dpp(0, upto, 0x112, 0xF, 0xF, true);
        upto += (int)__builtin_amdgcn_update_dpp(0, upto, 0x114, 0xF, 0xF, true);
        upto += (int)__builtin_amdgcn_update_dpp(0, upto, 0x118, 0xF, 0xF, true);
        const int s0 = __builtin_amdgcn_readlane(upto, 15), s1 = s0 + __builtin_amdgcn_readlane(upto, 31), s2 = s1 + __builtin_amdgcn_readlane(upto, 47);
        upto += lane < 16 ? 0 : lane < 32 ? s0 : lane < 48 ? s1 : s2;
        const uint64_t past = __ballot(before + upto > u);
        if (past) {
            const int l = __builtin_ctzll(past);
            const int k = u - before - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(n, l));
            if (k < 0 || k >= __builtin_amdgcn_readlane(n, l))  // ends that decrease: their rows may add up beyond 32 bits
                return {0, 0, 0};
            return {e0 + l, __builtin_amdgcn_readlane(begin, l) + k * R, min(__builtin_amdgcn_readlane(rows, l) - k * R, R)};
        }
        before += __builtin_amdgcn_readlane(upto, 63);
        last_end = __builtin_amdgcn_readlane(end, 63);
    }
    return {0, 0, 0};
}

// XR rows of x (up to 16, or a multiple of it); NT tiles of 16 rows of W a wavefront; WK wavefronts along K, the others along N. U units (4,
// 2 or 1) are loaded at a time.
template <int XR, int NT, int WK, int U, bool TILED, bool GROUPED>
__global__ __launch_bounds__(kGemvThreads) void fp4_gemv_kernel(const uint8_t *__restrict__ x, int64_t ldx_bytes, GemvRows map,
                                                                const uint8_t *__restrict__ w_q, const uint8_t *__restrict__ w_s, int M, int N, int nb,
                                                                uint32_t blocks_n, uint8_t *__restrict__ c, bool c_bf16, int64_t ldc, bool c_vector)
{
    constexpr int R = XR, MT = (XR + 15) / 16, WN = kGemvWaves / WK;
    constexpr int LANES = 16 * U;             // lanes of a row of x in a load
    constexpr int XL = XR * LANES > 64 ? XR * LANES / 64 : 1;  // loads of x
    // LDS of a wavefront, in pieces of 16 bytes: x [row][unit][16], W [tile][unit][row][4], scales [tile][row] (the dwords of four units)
    constexpr int XP = XR * LANES > 64 ? XR * LANES : 64, WP = NT * U * 64;
    __shared__ uint4 staged[kGemvWaves][XP + WP + NT * 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int wk = wave % WK, wn = wave / WK;
    const uint32_t block = blockIdx.x % blocks_n, u_piece = blockIdx.x / blocks_n;
    GemvPiece p;
    if constexpr (GROUPED)
        p = grouped_piece<R>(map.ends, map.groups, M, (int)u_piece, lane);
    else
        p = {0, (int)u_piece * R, min(M - (int)u_piece * R, R)};
    if (p.count <= 0)
        return;

    // ---- rows of W: four lanes a row, from block 4u + lane % 4 on; scales of the next four units, one dword a lane
    const int n0 = ((int)block * WN + wn) * NT * 16;
    const int s_unit = TILED ? g : lane & 3, s_row = TILED ? r : lane >> 2;
    const uint8_t *wq[NT], *ws[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int w_row = min(n0 + t * 16 + (lane >> 2), N - 1), s_n = min(n0 + t * 16 + s_row, N - 1);
        wq[t] = w_q + p.expert * (GROUPED ? map.wq_group_bytes : 0) + w_row * ((int64_t)nb * 16) + (lane & 3) * 16;
        ws[t] = w_s + p.expert * (GROUPED ? map.ws_group_bytes : 0) + (TILED ? ((int64_t)(s_n >> 6) * ((nb + 3) / 4) * 64 + (s_n & 63)) * 4 : (int64_t)s_n * nb);
    }

    struct Units {
        uint4 w[NT][U], x[XL];
        uint32_t s[NT];
    };
    const int whole = nb / kUnit, begin = (int)((int64_t)whole * wk / WK), end = (int)((int64_t)whole * (wk + 1) / WK);
    auto load_w = [&](Units &d, int u) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int j = 0; j < U; ++j)
                d.w[t][j] = stream_load(reinterpret_cast<const uint4 *>(wq[t] + (int64_t)min(u + j, end - 1) * 64));
            __builtin_memcpy(&d.s[t], ws[t] + (int64_t)min(u + s_unit, end - 1) * (TILED ? 256 : 4), 4);
        }
        MXFP8_PIN();
    };
    // The first weights are requested before the rows of x are worked out: 6.2 -> 5.5 us for 16 rows of a 4096 x 4096 matrix. With
    // experts the entries of the plan go first, or their rows of x wait behind the weights: 6.4 us, against 6.9, for 8 experts' 2048 x 1408.
    Units d;
    if (!GROUPED && begin < end)
        load_w(d, begin);

    // ---- rows of x of the columns that this lane has of C (-1: zeros), and of the pieces that it loads
    int at[MT];
    uint64_t any = 0;
    int first_row = 0;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        at[t] = t * 16 + r < p.count ? p.first + t * 16 + r : -1;
        if (GROUPED && map.sources && at[t] >= 0) {
            const uint32_t i = (uint32_t)map.sources[at[t]];
            at[t] = i < map.entries ? (int)(i / map.slots) : -1;
        }
        const uint64_t given = __ballot(at[t] >= 0);
        if (!any && given)
            first_row = __builtin_amdgcn_readlane(at[t], (int)__builtin_ctzll(given));
        any |= given;
    }
    const int lane_row = lane / LANES, lane_piece = lane % LANES;
    const uint8_t *xp[XL];
#pragma unroll
    for (int q = 0; q < XL; ++q) {
        const int m = q * (64 / LANES);  // the first of the rows of load q; they lie in one tile
        const int row = U == 4 ? __builtin_amdgcn_readlane(at[m / 16], m % 16) : __shfl(at[m / 16], (m + lane_row) % 16, 64);
        xp[q] = x + (row < 0 ? first_row : row) * ldx_bytes + lane_piece * 16;
    }
    uint4 *const lds_x = staged[wave], *const lds_w = lds_x + XP;
    uint32_t *const lds_s = reinterpret_cast<uint32_t *>(lds_w + WP);
    v4f acc[NT][MT] = {};
    auto load_x = [&](Units &d, int u) __attribute__((always_inline)) {
        const int last = (end - u) * 16 - 1;  // pieces of x behind the last unit are not multiplied: any others will do
#pragma unroll
        for (int q = 0; q < XL; ++q)
            d.x[q] = *reinterpret_cast<const uint4 *>(xp[q] + (int64_t)u * 256 + (lane_piece <= last ? 0 : -(lane_piece & ~15) * 16));
        MXFP8_PIN();
    };
    // Places are XORed so that the sixteen lanes that are served together hit different banks.
    auto stage = [&](const Units &d) __attribute__((always_inline)) {
        MXFP8_FENCE();
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int q = 0; q < XL; ++q) {
            const int m = q * (64 / LANES) + lane_row;
            if (XR * LANES >= 64 || m < XR)
                lds_x[m * LANES + (lane_piece ^ (m & 15))] = d.x[q];
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int j = 0; j < U; ++j)
                lds_w[(t * U + j) * 64 + (lane & ~3) + ((lane ^ (lane >> 4)) & 3)] = d.w[t][j];
            lds_s[t * 64 + s_row * 4 + s_unit] = d.s[t];
        }
        __builtin_amdgcn_wave_barrier();
        MXFP8_FENCE();
    };
    auto multiply = [&](int count) __attribute__((always_inline)) {
        uint32_t s[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint4 scales = *reinterpret_cast<const uint4 *>(lds_s + t * 64 + r * 4);
            s[t][0] = scales.x, s[t][1] = scales.y, s[t][2] = scales.z, s[t][3] = scales.w;
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (j >= count)
                break;
            v8bf a[NT][4];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const uint4 w = lds_w[(t * U + j) * 64 + r * 4 + (g ^ (r >> 2))];
                const float scale = scale_operand((s[t][j] >> (8 * g)) & 0xFFu);
                a[t][0] = fp4_word_bf16(w.x, scale), a[t][1] = fp4_word_bf16(w.y, scale);
                a[t][2] = fp4_word_bf16(w.z, scale), a[t][3] = fp4_word_bf16(w.w, scale);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const int m = min(t * 16 + r, XR - 1);
                    const v8bf b = __builtin_bit_cast(v8bf, lds_x[m * LANES + ((j * 16 + 4 * g + i) ^ (m & 15))]);
#pragma unroll
                    for (int k = 0; k < NT; ++k)
                        acc[k][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[k][i], b, acc[k][t], 0, 0, 0);
                }
        }
        MXFP8_PIN();
    };
    // The next units are on their way while those in LDS are multiplied.
    if (any && begin < end) {
        if (GROUPED)
            load_w(d, begin);
        load_x(d, begin);
        for (int u = begin; u < end; u += U) {
            stage(d);
            if (u + U < end) {
                load_w(d, u + U);
                load_x(d, u + U);
            }
            multiply(end - u);
        }
    }
    if (any && nb % kUnit && wk == WK - 1) {  // one to three blocks behind the whole units
        const int rest = nb % kUnit;
        d = {};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if ((lane & 3) < rest)
                d.w[t][0] = *reinterpret_cast<const uint4 *>(wq[t] + (int64_t)whole * 64);
            if (s_unit == 0)
                for (int b = 0; b < rest; ++b)
                    d.s[t] |= (uint32_t)ws[t][(int64_t)whole * (TILED ? 256 : 4) + b] << (8 * b);
        }
        if (lane_piece < rest * 4)
#pragma unroll
            for (int q = 0; q < XL; ++q)
                d.x[q] = *reinterpret_cast<const uint4 *>(xp[q] + (int64_t)whole * 256);
        stage(d);
        multiply(1);
    }

    // ---- sums of the wavefronts along K, in their order; wavefront k of them then stores the tiles k, k + WK, ... of NT x MT
    if constexpr (WK > 1) {
        static_assert(NT * MT * 64 <= XP + WP, "the sums take the place of what is staged");
        MXFP8_FENCE();
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int k = 0; k < NT * MT; ++k)
            reinterpret_cast<v4f *>(staged[wave])[k * 64 + lane] = acc[k / MT][k % MT];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NT * MT; ++k)
            if (k % WK == wk) {
                v4f sum = reinterpret_cast<const v4f *>(staged[wn * WK])[k * 64 + lane];
#pragma unroll
                for (int w = 1; w < WK; ++w)
                    sum += reinterpret_cast<const v4f *>(staged[wn * WK + w])[k * 64 + lane];
                acc[k / MT][k % MT] = sum;
            }
    }
#pragma unroll
    for (int k = 0; k < NT * MT; ++k) {
        const int m = k % MT * 16 + r, n = n0 + k / MT * 16 + 4 * g;
        if ((WK > 1 && k % WK != wk) || m >= p.count || n >= N)
            continue;
        const v4f sum = GROUPED && at[k % MT] < 0 ? v4f{0, 0, 0, 0} : acc[k / MT][k % MT];
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
}

// Pieces of at most R rows that the rows of C are cut into: an expert's rows take at most one more than they fill.
static int64_t gemv_pieces(const GemvRows &map, int64_t M, int R)
{
    const int64_t some = map.ends ? min((int64_t)map.groups, M) : 0;
    return map.ends ? some + (M - some) / R : (M + R - 1) / R;
}

template <int XR, int NT, int WK, int U, bool TILED>
static hipError_t launch_fp4_gemv_t(const void *x, int64_t ldx, const GemvRows &map, const uint8_t *w_q, const uint8_t *w_s, int64_t M, int64_t N,
                                    int64_t K, void *c, bool c_bf16, int64_t ldc, hipStream_t stream)
{
    constexpr int COLS = kGemvWaves / WK * NT * 16;  // rows of W of a workgroup
    const int64_t pieces = gemv_pieces(map, M, XR);
    const int64_t blocks_n = (N + COLS - 1) / COLS;
    if (blocks_n * pieces > kMostGemvWorkgroups)
        return hipErrorInvalidConfiguration;
    const bool vector = reinterpret_cast<uintptr_t>(c) % 16 == 0 && (ldc * (c_bf16 ? 2 : 4)) % 16 == 0;
    auto kern = map.ends ? fp4_gemv_kernel<XR, NT, WK, U, TILED, true> : fp4_gemv_kernel<XR, NT, WK, U, TILED, false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)(blocks_n * pieces)), dim3(kGemvThreads), 0, stream, static_cast<const uint8_t *>(x), ldx * 2, map, w_q, w_s,
                       (int)M, (int)N, (int)(K / kBlock), (uint32_t)blocks_n, static_cast<uint8_t *>(c), c_bf16, ldc, vector);
    return hipGetLastError();
}

template <int XR, int NT, int U, bool TILED>
static hipError_t launch_fp4_gemv_rows(const void *x, int64_t ldx, const GemvRows &map, const uint8_t *w_q, const uint8_t *w_s, int64_t M, int64_t N,
                                       int64_t K, void *c, bool c_bf16, int64_t ldc, hipStream_t stream)
{
    // As many wavefronts along K as have four units each, up to what the LDS lets be resident: 2048 with 16 rows of x and more, else some
    // 8192. In us with 1 | 2 | 4 | 8 along K: [1 x 4096 x 14336] 40.7 | 22.5 | 13.8 | 10.7, [1 x 28672 x 4096] 14.4 | 16.7 | 15.8 | 16.4,
    // [64 x 28672 x 4096] 71.4 | 43.8 | 50.7 | 55.1, 48 tokens x 4 of 64 experts [5632 x 2048] 78.7 | 75.1 | 83.6 | 107.7.
    const int64_t tiles = (N + 16 * NT - 1) / (16 * NT) * gemv_pieces(map, M, XR), units = K / (kUnit * kBlock);
    const int64_t most = XR >= 16 ? 2048 : 8192;
    int wk = 1;
    while (wk < kGemvWaves && units >= 8 * wk && (tiles * wk * 2 <= most || (NT > 1 && wk == 1)))
        wk *= 2;
    auto launch = wk == 1   ? launch_fp4_gemv_t<XR, NT, 1, U, TILED>
                  : wk == 2 ? launch_fp4_gemv_t<XR, NT, 2, U, TILED>
                  : wk == 4 ? launch_fp4_gemv_t<XR, NT, 4, U, TILED>
                            : launch_fp4_gemv_t<XR, NT, 8, U, TILED>;
    return launch(x, ldx, map, w_q, w_s, M, N, K, c, c_bf16, ldc, stream);
}

hipError_t launch_fp4_gemv(const void *x, int64_t tokens, int64_t ldx, const int32_t *sources, int slots, const uint8_t *w_q, const uint8_t *w_s,
                           const int32_t *group_ends, int groups, int64_t ws_group_bytes, int64_t M, int64_t N, int64_t K, void *c, bool c_bf16,
                           int64_t ldc, bool tiled_scales, hipStream_t stream)
{
    const GemvRows map = {sources, (uint32_t)(tokens * slots), (uint32_t)slots, group_ends, groups, N * (K / 2), ws_group_bytes};
    // Rows that an expert is made ready for: what it has in the mean is known, and the ones that are chosen have more than that.
    const int64_t rows = !group_ends ? M : M == 1 || (sources && tokens == 1) ? 1 : (M + groups - 1) / groups * 3 / 2 + 1;
    auto launch = [&](auto tiled) {
        constexpr bool T = decltype(tiled)::value;
        // Two or four tiles of W a wavefront, so that x is fetched and reordered for more of them, where there are tiles enough (of 16
        // rows of W and the XR rows of a piece). In us, one tile | two | four: [8 x 28672 x 4096] 22.2 | 19.2, [64 x 28672 x 4096]
        // 73.2 | 50.9 | 43.8, [64 x 4096 x 4096] 12.2 | 10.2 | 13.7, [32 x 4096 x 4096] 7.9 | 9.6 | 12.5, [8 x 4096 x 4096] 5.2 | 6.2.
        const int64_t n16 = (N + 15) / 16;
        auto tiles = [&](int xr) { return n16 * gemv_pieces(map, M, xr); };
        auto pick = rows <= 1    ? launch_fp4_gemv_rows<1, 1, 4, T>
                    : rows <= 4  ? launch_fp4_gemv_rows<4, 1, 4, T>
                    : rows <= 8  ? (tiles(8) < 1024 ? launch_fp4_gemv_rows<8, 1, 2, T> : launch_fp4_gemv_rows<8, 2, 2, T>)
                    : rows <= 16 ? (tiles(16) < 1024 ? launch_fp4_gemv_rows<16, 1, 2, T> : launch_fp4_gemv_rows<16, 2, 2, T>)
                    : tiles(32) < 512  ? launch_fp4_gemv_rows<32, 1, 1, T>
                    : tiles(32) < 2048 ? launch_fp4_gemv_rows<32, 2, 1, T>
                                       : launch_fp4_gemv_rows<32, 4, 1, T>;
        return pick(x, ldx, map, w_q, w_s, M, N, K, c, c_bf16, ldc, stream);
    };
    return tiled_scales ? launch(std::true_type{}) : launch(std::false_type{});
}

}  // namespace mxfp8
