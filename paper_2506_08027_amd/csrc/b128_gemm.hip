// Products of E4M3 operands with an FP32 scale for each block of 128 (include/mxfp8_b128.h): C[m, n] = sum_b sa[b, m] sb[b, n] P_b[m, n],
// P_b the sum of block b's 128 products.
//
// One v_mfma_f32_16x16x128_f8f6f4 makes P_b of a 16 x 16 tile from a zero accumulator, and four FMAs a lane add it, scaled, to the sums
// (32 cycles of the matrix pipe, 16 of the vector pipe). The sums have to lie in ordinary registers for that: a wavefront's tile is
// 128 x 64 at most, two wavefronts a SIMD. B is fed as the first operand and A as the second, so that a lane's four sums are one row of
// C: with B cut into tiles one factor sa sb per row and step serves them all; with B cut into vectors each column has its own, and the
// vector pipe as much to do as the matrix pipe.
//   That instruction cuts every product of eight neighbouring k off at 2^-13 of the largest of them (mfma_model.py of the tests): some 2^-16 of
// a result, far below the rounding of a BF16 one. FP32 results have to be better than that: there the codes are widened to BF16, which is
// exact, and four v_mfma_f32_16x16x32_bf16 make P_b with FP32 roundings alone, at half the rate. [14336 x 4096 x 8192] 860 us = 1.12 PFLOP/s (matrix
// pipes busy in 51 % of the cycles: widening takes the vector pipe) where the FP8 instruction took 526 (relative error over ordinary data 1.5e-7 instead of 1.5e-5; an FP32 library product of the decoded operands has 1.5e-6).
//   Operands and A's scales go to LDS without passing through registers, a ring of S steps of 128 k. LDS rows are 128 bytes; the 16-byte
// chunk index is XORed with (row / 2) % 8, on the global side, so that the 16 lanes of a fragment read hit different banks (the layout of
// fragments and of the matrix instruction is described in gemm.hip).
//   The last step of a K that 128 does not divide: chunks that are not there are read from the row's first chunk of the step, and A's
// fragments are zero there.
//   Measured: [8192 x 14336 x 4096] 413 us = 2.33 PFLOP/s, weight gradient [14336 x 4096 x 8192] 516 us = 1.86 (BF16 out; with the same operands
// again and again 394 and 484). What bounds it there: the matrix pipes are busy in 60 and 43 % of the cycles (61 % of those of [4096 x 4096 x 16384]), and the card holds its power by running
// at 1.92 GHz: that last product takes 235 us, 189 with zeros for operands. The product whose scales the matrix instruction applies itself
// (MXFP8) takes 195 and 166. [96 x 4096 x 14336] 19.3 us: 60 MB of operands, the sums of four parts, a second launch.
#include "b128_launches.h"
#include "gemm_device.h"

#include <type_traits>

namespace mxfp8 {

constexpr int kWide = 128;  // values of a block

template <int BM_, int BN_, int WAVES_M_, int WAVES_N_, int STAGES_> struct WideCfg {
    static constexpr int BM = BM_, BN = BN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, STAGES = STAGES_;
    static constexpr int WAVES = WAVES_M * WAVES_N, THREADS = 64 * WAVES;
    static constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N, TM = WM / 16, TN = WN / 16;
    static constexpr int DATA_BYTES = (BM + BN) * BK;
    static constexpr int A_LOADS = BM / 8 / WAVES, B_LOADS = BN / 8 / WAVES, LOADS = A_LOADS + B_LOADS;  // 8-row requests per wavefront and step
    // 64 scales a request: A's, then B's where it is cut into vectors; some are made twice
    static constexpr int AG = (BM + 63) / 64, BG = (BN + 63) / 64;
    static constexpr int scale_groups(bool vectors) { return AG + (vectors ? BG : 0); }
    static constexpr int scale_loads(bool vectors) { return (scale_groups(vectors) + WAVES - 1) / WAVES; }
    static constexpr int stage_bytes(bool vectors) { return DATA_BYTES + scale_groups(vectors) * 256; }
    static constexpr int PITCH = WN * 4 + 32;  // staged row of the epilogue
    static constexpr int lds_bytes(bool vectors)
    {
        const int ring = STAGES * stage_bytes(vectors), epilogue = WAVES * 16 * PITCH;
        return ring > epilogue ? ring : epilogue;
    }
    static_assert(WM % 16 == 0 && WN % 16 == 0 && BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "whole instructions and requests");
    static_assert(128 % WN == 0, "a wavefront's columns lie in one tile of B's scales");
};

// Four consecutive columns of a row of C, or as many as there are
template <bool OUT_BF16> __device__ __forceinline__ void store_some(uint8_t *to, const v4f &v, int count)
{
    for (int e = 0; e < 4; ++e)
        if (e < count) {
            if constexpr (OUT_BF16)
                reinterpret_cast<__bf16 *>(to)[e] = (__bf16)v[e];
            else
                reinterpret_cast<float *>(to)[e] = v[e];
        }
}

// Codes of a fragment as four operands of the BF16 matrix instruction (exact)
struct WideFragment {
    v8bf k[4];
};
__device__ __forceinline__ WideFragment widened(const v8i &codes)
{
    WideFragment f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[2 * i], 1.0f, false),
                   b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[2 * i], 1.0f, true),
                   c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[2 * i + 1], 1.0f, false),
                   d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[2 * i + 1], 1.0f, true);
        f.k[i] = v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    return f;
}

// Part `p` of `parts` of the steps of K; with parts > 1 the sums go to c (FP32) at p * part_bytes. EXACT: codes are multiplied as BF16.
template <class Cfg, bool OUT_BF16, bool VECTORS, bool EXACT>
__global__ __launch_bounds__(Cfg::THREADS, 2) void b128_gemm_kernel(const uint8_t *__restrict__ a_q, int64_t lda, const float *__restrict__ a_s,
                                                                 const uint8_t *__restrict__ b_q, int64_t ldb, const float *__restrict__ b_s, int M, int N,
                                                                 int K, uint8_t *__restrict__ c, int64_t ldc_bytes, int tiles_m, int tiles_n, int parts,
                                                                 int64_t part_bytes, bool vec_store)
{
    MXFP8_DYNAMIC_LDS(lds);
    constexpr int TM = Cfg::TM, TN = Cfg::TN, S = Cfg::STAGES, STAGE = Cfg::stage_bytes(VECTORS);
    constexpr int SREQ = Cfg::scale_loads(VECTORS), SGROUPS = Cfg::scale_groups(VECTORS), L = Cfg::LOADS + SREQ;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / Cfg::WAVES_N, wn = wave % Cfg::WAVES_N;
    const int r16 = lane & 15, g = lane >> 4;
    const int KB = (K + BK - 1) / BK;
    const uint32_t lds_base = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);

    const int ntiles = tiles_m * tiles_n, part = blockIdx.x / ntiles;
    int tile_m, tile_n;
    tile_of_block(blockIdx.x % ntiles, ntiles, tiles_m, tiles_n, tile_m, tile_n);
    const int m0 = tile_m * Cfg::BM, n0 = tile_n * Cfg::BN;
    const int begin = (int)((int64_t)KB * part / parts), end = (int)((int64_t)KB * (part + 1) / parts);
    c += part * part_bytes;

    // ---- requests: 8-row groups of A's rows of the tile and of B's
    const int ld_r = lane >> 3, ld_c = lane & 7;
    int tail = ((K + 15) >> 4) - (KB - 1) * 8;  // chunks of the last step
    const uint8_t *const a_src = a_q + (int64_t)m0 * lda, *const b_src = b_q + (int64_t)n0 * ldb;
    uint32_t goff[Cfg::LOADS], back[2][2];
    auto group = [&](int q) __attribute__((always_inline)) { return q < Cfg::A_LOADS ? wave * Cfg::A_LOADS + q : wave * Cfg::B_LOADS + q - Cfg::A_LOADS; };
#pragma unroll
    for (int q = 0; q < Cfg::LOADS; ++q) {
        const bool of_a = q < Cfg::A_LOADS;
        const int row = group(q) * 8 + ld_r;
        // rows behind the last one re-read it
        goff[q] = (uint32_t)min(row, (of_a ? M - m0 : N - n0) - 1) * (uint32_t)(of_a ? lda : ldb) + (ld_c ^ ((row >> 1) & 7)) * 16;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // in odd and even requests of A and of B: from a chunk that the last step has not to its first one
        const int chunk = ld_c ^ ((group(i < 2 ? i : Cfg::A_LOADS + i - 2) * 4 + (ld_r >> 1)) & 7);
        back[i >> 1][i & 1] = chunk < tail ? 0 : chunk * 16;
    }
    const float *ssrc[SREQ];
    uint32_t soff[SREQ];
    int64_t sstep[SREQ];
#pragma unroll
    for (int j = 0; j < SREQ; ++j) {
        const int grp = (wave + j * Cfg::WAVES) % SGROUPS;  // wavefront-uniform
        const bool of_a = grp < Cfg::AG;
        const int first = of_a ? m0 : n0, row = (of_a ? grp : grp - Cfg::AG) * 64 + lane;
        ssrc[j] = (of_a ? a_s : b_s) + first;
        soff[j] = (uint32_t)min(row, (of_a ? M : N) - first - 1) * 4;
        sstep[j] = of_a ? M : N;
    }
    // request q of step kt into a slot
    auto issue = [&](int q, int kt, int slot) __attribute__((always_inline)) {
        const uint32_t stage = lds_base + slot * STAGE;
        if (q < Cfg::LOADS) {
            const uint32_t ragged = kt == KB - 1 ? ~0u : 0u;
            const bool of_a = q < Cfg::A_LOADS;
            dma_load<16>((of_a ? a_src : b_src) + (int64_t)kt * BK, goff[q] - (back[of_a ? 0 : 1][(of_a ? q : q - Cfg::A_LOADS) & 1] & ragged),
                         stage + (of_a ? 0 : Cfg::BM * BK) + group(q) * 1024);
        } else {
            const int j = q - Cfg::LOADS;
            dma_load<4>(reinterpret_cast<const uint8_t *>(ssrc[j] + kt * sstep[j]), soff[j], stage + Cfg::DATA_BYTES + (wave + j * Cfg::WAVES) % SGROUPS * 256);
        }
    };

    // fragment addresses inside a stage
    const int a_row = wm * Cfg::WM + r16, b_row = wn * Cfg::WN + r16;
    const int a_off0 = a_row * BK + ((g ^ ((a_row >> 1) & 7)) << 4), a_off1 = a_row * BK + (((4 + g) ^ ((a_row >> 1) & 7)) << 4);
    const int b_off0 = (Cfg::BM + b_row) * BK + ((g ^ ((b_row >> 1) & 7)) << 4), b_off1 = (Cfg::BM + b_row) * BK + (((4 + g) ^ ((b_row >> 1) & 7)) << 4);
    auto fragment = [&](const uint8_t *stage, int off0, int off1) __attribute__((always_inline)) {
        const v4i lo = *reinterpret_cast<const v4i *>(stage + off0), hi = *reinterpret_cast<const v4i *>(stage + off1);
        return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    const int tile_row = min(n0 + wn * Cfg::WN, N - 1) / kWide;  // B cut into tiles: row of this wavefront's scales
    const float *const b_tiles = b_s + (int64_t)tile_row * KB;

    v4f acc[TM][TN] = {};
    // Fragments of A of half the row groups: the other half's, and the next step's, take their places as they are used up.
    constexpr int H = TM / 2, SETS = EXACT ? TM : H > 1 ? H : 2;
    v8i fa[SETS], fb[TN];
    v4f cols[VECTORS ? TN : 1];
    float tile_scale = 1.0f, row_scale[SETS];
    auto read_a = [&](int kt, int i) __attribute__((always_inline)) {
        const uint8_t *const stage = lds + kt % S * STAGE;
        fa[i % SETS] = fragment(stage, a_off0 + i * 2048, a_off1 + i * 2048);
        row_scale[i % SETS] = reinterpret_cast<const float *>(stage + Cfg::DATA_BYTES)[wm * Cfg::WM + r16 + i * 16];
    };
    auto read_b = [&](int kt, int j) __attribute__((always_inline)) {
        const uint8_t *const stage = lds + kt % S * STAGE;
        fb[j] = fragment(stage, b_off0 + j * 2048, b_off1 + j * 2048);
        if constexpr (VECTORS)
            cols[j] = *reinterpret_cast<const v4f *>(stage + Cfg::DATA_BYTES + Cfg::AG * 256 + (wn * Cfg::WN + 4 * g + j * 16) * 4);
    };
    // One step: the first half of the row groups row by row, the other half column by column, so that what is read from LDS is spread
    // over the step: behind each row the row group that takes its place, behind each column B's fragment of the next step, behind each
    // row group's last column A's of the next step. In front of the second column there everything of this step has been read and the
    // next one's has arrived: from there on the requests of step kt + S (the last one's again where there is none, so that all steps are
    // alike) go to this one's slot, spread too: all at once they wait for the address unit, and the matrix instructions behind them.
    constexpr int MMAS = TM * TN, FREE = H * TN + H;  // matrix instructions, and those in front of the barrier
    constexpr int P = H >= 2 ? 3 : 2;                  // sums of blocks that are under way
    auto step = [&](int kt, auto last) __attribute__((always_inline)) {
        constexpr bool LAST = decltype(last)::value, NEXT = !LAST;
        const float tiles = tile_scale;
        v4f p[P];
        float scale[SETS];
        auto row_of = [](int m) constexpr { return m < H * TN ? m / TN : H + (m - H * TN) % H; };
        auto col_of = [](int m) constexpr { return m < H * TN ? m % TN : (m - H * TN) / H; };
        auto add = [&](int m) __attribute__((always_inline)) {  // matrix instruction m of the step
            const int i = row_of(m), j = col_of(m);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                // the scales' product first: the sum times one of them alone can leave FP32, and this waits for no matrix instruction
                acc[i][j][e] = __builtin_fmaf(p[m % P][e], VECTORS ? cols[VECTORS ? j : 0][e] * scale[i % SETS] : scale[i % SETS], acc[i][j][e]);
            // with that, column j is done with its fragment and scales
            if (NEXT && i == TM - 1)
                read_b(kt + 1, j);
        };
#pragma unroll
        for (int m = 0; m < MMAS; ++m) {
            const int i = row_of(m), j = col_of(m);
            if (m == FREE && NEXT) {
                MXFP8_FENCE();
                MXFP8_WAIT_VMCNT_AND_LDS((S - 2) * L);
                MXFP8_BARRIER();
                MXFP8_FENCE();
                if (!VECTORS)
                    tile_scale = scalar_load(b_tiles + kt + 1);
            }
            if (j == 0 && LAST) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    fa[i % SETS][e] = (e < 4 ? g : 4 + g) < tail ? fa[i % SETS][e] : 0;
            }
            p[m % P] = mfma_e4m3(fb[j], fa[i % SETS], v4f{0.f, 0.f, 0.f, 0.f});
            MXFP8_PIN();
            if (m >= P - 1)
                add(m - (P - 1));
            if (j == 0)  // (not before: that sum may be of the row group whose place this one has taken)
                scale[i % SETS] = row_scale[i % SETS] * tiles;
            if (i < H && j == TN - 1)
                read_a(kt, i + H);
            if (NEXT && i >= H && j == TN - 1)
                read_a(kt + 1, i - H);
            if (NEXT && m >= FREE) {
#pragma unroll
                for (int q = (m - FREE) * L / (MMAS - FREE); q < (m + 1 - FREE) * L / (MMAS - FREE); ++q)
                    issue(q, min(kt + S, end - 1), kt % S);
            }
            MXFP8_PIN();
        }
#pragma unroll
        for (int m = MMAS - (P - 1); m < MMAS; ++m)
            add(m);
        MXFP8_PIN();
    };
    // One step with exact products: all fragments are read at once, so that the slot is free behind a barrier, B's are widened for the whole
    // step and A's row group by row group. Two workgroups a unit cover each other's waits.
    auto exact_step = [&](int kt, auto last) __attribute__((always_inline)) {
        constexpr bool LAST = decltype(last)::value;
        const float tiles = VECTORS ? 1.0f : scalar_load(b_tiles + kt);
        WideFragment b[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j)
            read_b(kt, j);
#pragma unroll
        for (int i = 0; i < TM; ++i)
            read_a(kt, i);
        if constexpr (!LAST) {
            MXFP8_FENCE();
            MXFP8_WAIT_VMCNT_AND_LDS(63);  // (the reads have returned)
            MXFP8_BARRIER();
            MXFP8_FENCE();
#pragma unroll
            for (int q = 0; q < L; ++q)
                issue(q, min(kt + S, end - 1), kt % S);
        }
#pragma unroll
        for (int j = 0; j < TN; ++j)
            b[j] = widened(fb[j]);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            if constexpr (LAST)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    fa[i][e] = (e < 4 ? g : 4 + g) < tail ? fa[i][e] : 0;
            const WideFragment a = widened(fa[i]);
            const float scale = row_scale[i] * tiles;
            v4f p[TN] = {};
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    p[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j].k[k], a.k[k], p[j], 0, 0, 0);
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[i][j][e] = __builtin_fmaf(p[j][e], VECTORS ? cols[VECTORS ? j : 0][e] * scale : scale, acc[i][j][e]);
        }
        if constexpr (!LAST) {
            MXFP8_FENCE();
            MXFP8_WAIT_VMCNT((S - 1) * L);
            MXFP8_BARRIER();
            MXFP8_FENCE();
        }
    };
    // ---- steps begin .. end - 1. Straight-line bodies: one that branches inside makes the compiler move the sums between registers.
    if (begin < end) {
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int q = 0; q < L; ++q)
                issue(q, min(begin + s, end - 1), (begin + s) % S);
        MXFP8_WAIT_VMCNT_AND_LDS((S - 1) * L);
        MXFP8_BARRIER();
        MXFP8_FENCE();
        if constexpr (!EXACT) {
            if (!VECTORS)
                tile_scale = scalar_load(b_tiles + begin);
#pragma unroll
            for (int i = 0; i < H; ++i)
                read_a(begin, i);
#pragma unroll
            for (int j = 0; j < TN; ++j)
                read_b(begin, j);
        }
        auto any_step = [&](int kt, auto last) __attribute__((always_inline)) {
            if constexpr (EXACT)
                exact_step(kt, last);
            else
                step(kt, last);
        };
        int kt = begin;
        for (; kt + 1 < end; ++kt)
            any_step(kt, std::false_type{});
        tail = kt == KB - 1 ? tail : 8;
        any_step(kt, std::true_type{});
        MXFP8_WAIT_VMCNT(0);
    }

    // ---- epilogue: 16-row groups through a wavefront-private LDS area (the ring is done with), whole rows out
    constexpr int ESZ = OUT_BF16 ? 2 : 4;
    MXFP8_FENCE();
    __syncthreads();
    const int mw = m0 + wm * Cfg::WM, nw = n0 + wn * Cfg::WN;  // first row and column of this wavefront
    if (vec_store) {
        constexpr int ROWB = Cfg::WN * ESZ, PITCH = ROWB + 32, CHUNKS = ROWB / 16;
        uint8_t *const area = lds + wave * 16 * Cfg::PITCH;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
                store_some<OUT_BF16>(area + r16 * PITCH + (j * 16 + 4 * g) * ESZ, acc[i][j], 4);
            MXFP8_FENCE();
            __builtin_amdgcn_wave_barrier();  // the reads below see the other lanes' writes (LDS serves a wavefront in order)
#pragma unroll
            for (int t = 0; t < (16 * CHUNKS + 63) / 64; ++t) {
                const int piece = t * 64 + lane, row = piece / CHUNKS, colb = piece % CHUNKS * 16;
                const int m = mw + i * 16 + row, n = nw + colb / ESZ;
                if ((16 * CHUNKS % 64 == 0 || piece < 16 * CHUNKS) && m < M && n < N) {
                    const uint8_t *const from = area + row * PITCH + colb;
                    uint8_t *const out = c + (int64_t)m * ldc_bytes + (int64_t)n * ESZ;
                    if (n + 16 / ESZ <= N) {
                        *reinterpret_cast<uint4 *>(out) = *reinterpret_cast<const uint4 *>(from);
                    } else {  // the row ends inside this piece
                        for (int e = 0; n + e < N; ++e)
                            if constexpr (OUT_BF16)
                                reinterpret_cast<uint16_t *>(out)[e] = reinterpret_cast<const uint16_t *>(from)[e];
                            else
                                reinterpret_cast<uint32_t *>(out)[e] = reinterpret_cast<const uint32_t *>(from)[e];
                    }
                }
            }
            MXFP8_FENCE();
            __builtin_amdgcn_wave_barrier();  // the next row group overwrites the area after these reads
        }
    } else {
#pragma unroll
        for (int i = 0; i < TM; ++i)
            if (mw + i * 16 + r16 < M)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const int n = nw + j * 16 + 4 * g;
                    store_some<OUT_BF16>(c + (int64_t)(mw + i * 16 + r16) * ldc_bytes + (int64_t)n * ESZ, acc[i][j], N - n);
                }
    }
}

// C = sum of the parts [parts][M][ld] in their order, rounded once; four columns a thread
template <bool OUT_BF16>
__global__ __launch_bounds__(256) void b128_join_kernel(const float *__restrict__ sums, int parts, int64_t part_elements, int64_t ld, int M, int N,
                                                        uint32_t quads, uint8_t *__restrict__ c, int64_t ldc_bytes, bool vec_store)
{
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = id / quads;
    const int n = (int)(id % quads) * 4;
    if (m >= M)
        return;
    const float *at = sums + m * ld + n;
    v4f sum = *reinterpret_cast<const v4f *>(at);
    for (int p = 1; p < parts; ++p)
        sum += *reinterpret_cast<const v4f *>(at + p * part_elements);
    uint8_t *const to = c + m * ldc_bytes + (int64_t)n * (OUT_BF16 ? 2 : 4);
    if (vec_store && n + 4 <= N) {
        if constexpr (OUT_BF16) {
            const v2bf a = {(__bf16)sum[0], (__bf16)sum[1]}, b = {(__bf16)sum[2], (__bf16)sum[3]};
            *reinterpret_cast<uint2 *>(to) = make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
        } else {
            *reinterpret_cast<v4f *>(to) = sum;
        }
    } else {
        store_some<OUT_BF16>(to, sum, N - n);
    }
}

// Tiles, and what they were measured to take (us): a step of 128 k while every unit has its share of them, or only one workgroup where it
// can have two; and what comes on top for a tile, its first requests and its epilogue. The larger the tile, the less a unit reads from
// L2 and LDS for its matrix instructions: [8192 x 14336 x 4096] takes 412 | 463 | 491 | 592 us with the first four (BF16 out). But there
// have to be enough of them: [2048 x 4096 x 4096] 51 | 36 | 38 | 43, [1003 x 2880 x 5632] 61 | 41 | 33 | 27, the last 34,
// [256 x 4096 x 4096] 43 | 27 | 24 | 20 | 13. The figures are the forward product's; weight gradients, which take the same plan, are slower in large
// tiles: [14336 x 4096 x 8192] 423 us by these figures, 484 measured.
using WideHuge = WideCfg<256, 256, 2, 4, 2>;
using WideLarge = WideCfg<256, 128, 4, 2, 2>;
using WidePair = WideCfg<128, 128, 2, 2, 2>;  // two workgroups a unit
using WideDeep = WideCfg<128, 128, 2, 4, 4>;  // one, and three steps under way
using WideSmall = WideCfg<64, 64, 2, 2, 4>;   // two
struct WideCost {
    int bm, bn, per_unit;
    float step, alone, tile;
};
constexpr WideCost kWideCosts[] = {{256, 256, 1, 1.70f, 1.40f, 4.0f},
                                   {256, 128, 1, 0.89f, 0.75f, 4.0f},
                                   {128, 128, 2, 0.98f, 0.56f, 4.0f},
                                   {128, 128, 1, 0.51f, 0.47f, 4.3f},
                                   {64, 64, 2, 0.40f, 0.28f, 2.2f}};
constexpr int kUnits = 256;  // compute units of the device

struct WidePlan {
    int tile;   // its place in the list
    int parts;  // of K
};
// The plan that these figures say is the fastest. Where there are few tiles K is cut into parts, whose sums are written, read again and
// added up by a second launch (4 MB a us).
static WidePlan wide_plan(int64_t M, int64_t N, int64_t K)
{
    const int64_t steps = (K + BK - 1) / BK;
    WidePlan best = {0, 1};
    float least = 1e30f;
    for (int t = 0; t < (int)(sizeof(kWideCosts) / sizeof(kWideCosts[0])); ++t) {
        const WideCost &cost = kWideCosts[t];
        const int64_t tiles = (M + cost.bm - 1) / cost.bm * ((N + cost.bn - 1) / cost.bn), slots = kUnits * cost.per_unit;
        for (int parts : {1, 2, 3, 4, 6, 8, 12, 16}) {
            if (parts > 1 && (tiles * parts > slots || steps < 2 * parts))
                break;
            const float rounds = (float)(tiles * parts) / (float)slots;
            // (a last round that is not full runs faster than a full one)
            const float share = rounds <= 1.0f ? 1.0f : 0.5f * (rounds + (float)((tiles * parts + slots - 1) / slots));
            const float us = share * ((float)((steps + parts - 1) / parts) * (tiles * parts <= kUnits ? cost.alone : cost.step) + cost.tile) +
                             (parts > 1 ? 2.5f + (float)parts * (float)M * (float)N * 8e-6f / 4.0f : 0.0f);
            if (us < least) {
                least = us;
                best = {t, parts};
            }
        }
    }
    return best;
}

// Exact products: tiles of 128 x 128, or of 64 x 64 where those would leave half of the units without one. In us (fprop, wgrad) with 128 x 128 |
// 64 x 64: 1024 tiles 125, 131 | 179, 200 ([4096 x 4096 x 4096]), 184 tiles 56, 51 | 52, 59 ([1003 x 2880 x 5632]), 144 tiles 19.3, 18.2 | 19.0, 21.1
// ([1536 x 1536 x 1536]), 128 tiles 42, 38 | 28, 31 ([512 x 4096 x 4096]), 64 tiles 41, 37 | 20, 23 ([256 x 4096 x 4096]). 256 x 128 takes as long as
// 128 x 128 at the largest sizes (845, 858 | 828, 904 at [8192 x 14336 x 4096]) and longer elsewhere.
static bool exact_in_small_tiles(int64_t M, int64_t N, int parts) { return (M + 127) / 128 * ((N + 127) / 128) * parts <= kUnits / 2; }

int b128_gemm_parts(int64_t M, int64_t N, int64_t K) { return wide_plan(M, N, K).parts; }

template <class Cfg, bool OUT_BF16, bool VECTORS, bool EXACT>
static hipError_t launch_wide(const uint8_t *a_q, int64_t lda, const float *a_s, const uint8_t *b_q, int64_t ldb, const float *b_s, int64_t M, int64_t N,
                              int64_t K, void *c, int64_t ldc, int parts, int64_t part_elements, hipStream_t stream)
{
    constexpr int ESZ = OUT_BF16 ? 2 : 4;
    const int64_t tiles_m = (M + Cfg::BM - 1) / Cfg::BM, tiles_n = (N + Cfg::BN - 1) / Cfg::BN;
    if (tiles_m * tiles_n * parts > INT32_MAX)
        return hipErrorInvalidConfiguration;
    const bool vec = reinterpret_cast<uintptr_t>(c) % 16 == 0 && ldc * ESZ % 16 == 0;
    auto kern = b128_gemm_kernel<Cfg, OUT_BF16, VECTORS, EXACT>;
    constexpr int bytes = Cfg::lds_bytes(VECTORS);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(tiles_m * tiles_n * parts)), dim3(Cfg::THREADS), bytes, stream, a_q, lda, a_s, b_q, ldb, b_s, (int)M, (int)N,
                       (int)K, static_cast<uint8_t *>(c), ldc * ESZ, (int)tiles_m, (int)tiles_n, parts, part_elements * ESZ, vec);
    return hipGetLastError();
}

hipError_t launch_b128_gemm(const uint8_t *a_q, int64_t lda, const float *a_s, const uint8_t *b_q, int64_t ldb, const float *b_s, bool vectors_b,
                            int64_t M, int64_t N, int64_t K, void *c, bool c_bf16, int64_t ldc, float *workspace, hipStream_t stream)
{
    const WidePlan plan = wide_plan(M, N, K);
    const int64_t ld = (N + 3) / 4 * 4;
    auto with = [&](auto out_bf16, auto vectors, void *to, int64_t ld_to) {
        constexpr bool B = decltype(out_bf16)::value, V = decltype(vectors)::value;
        auto run = plan.tile == 0   ? launch_wide<WideHuge, B, V, false>
                   : plan.tile == 1 ? launch_wide<WideLarge, B, V, false>
                   : plan.tile == 2 ? launch_wide<WidePair, B, V, false>
                   : plan.tile == 3 ? launch_wide<WideDeep, B, V, false>
                                    : launch_wide<WideSmall, B, V, false>;
        if (!c_bf16)
            run = exact_in_small_tiles(M, N, plan.parts) ? launch_wide<WideSmall, false, V, true> : launch_wide<WidePair, false, V, true>;
        return run(a_q, lda, a_s, b_q, ldb, b_s, M, N, K, to, ld_to, plan.parts, M * ld, stream);
    };
    auto with_out = [&](auto vectors) {
        return plan.parts > 1 ? with(std::false_type{}, vectors, workspace, ld)
               : c_bf16       ? with(std::true_type{}, vectors, c, ldc)
                              : with(std::false_type{}, vectors, c, ldc);
    };
    const hipError_t e = vectors_b ? with_out(std::true_type{}) : with_out(std::false_type{});
    if (e != hipSuccess || plan.parts == 1)
        return e;
    const int64_t quads = ld / 4, esize = c_bf16 ? 2 : 4;
    const bool vec = reinterpret_cast<uintptr_t>(c) % (4 * esize) == 0 && ldc % 4 == 0;
    auto join = c_bf16 ? b128_join_kernel<true> : b128_join_kernel<false>;
    hipLaunchKernelGGL(join, dim3((unsigned)((M * quads + 255) / 256)), dim3(256), 0, stream, workspace, plan.parts, M * ld, ld, (int)M, (int)N,
                       (uint32_t)quads, static_cast<uint8_t *>(c), ldc * esize, vec);
    return hipGetLastError();
}

}  // namespace mxfp8
