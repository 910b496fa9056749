// A whole mixture-of-experts layer for a few tokens (include/mxfp8_layer.h) in two kernels: the up-projections with the gate, and the
// down-projections with the sum over a token's experts. The stream of a wavefront is described in few_rows.h.
//
// First kernel. A workgroup has some tiles of 16 of an expert's `inter` values, gate and other rows of W side by side, for all
// rows of the expert, up to XR at a time; it finds them in the router's choices by itself. Where there are fewer choices than experts
// a workgroup is made for each of them and those whose expert an earlier one has chosen too end at once. h times the router's
// weight goes to the workspace as BF16 planes, each the rest that those before it leave: rounded to one it would lose 2^-9, with two
// 2^-17 (BF16 results), with three 2^-25 (FP32 results).
// One more workgroup writes the plan of the second kernel: segments of up to XR2 rows of one expert.
// Second kernel. A workgroup has 16 columns of the output for all tokens and walks over the segments: their units of K make one
// sequence of which each of its wavefronts takes a contiguous part, its loads running on from one segment into the next. The wavefronts'
// sums for each token meet in LDS and are added in the order of the wavefronts.
// Tokens are taken 64 at a time (a chunk), each with its own workgroups.
// Where 16 columns a workgroup leave units idle, several share them and the one that arrives last adds up their sums.
// Measured in a captured graph, weights from HBM: 48 tokens x 4 of 64 experts, [2048 x 2816], scales for 128 x 128: 173 us, 6.1 TB/s, what
// a large read reaches (180 on another card); 4 x 8 [2048 x 1408], MXFP8: 51 (4.6). 1 x 8, MXFP4: 19 us for 37 MB. Of these 6.6 are two launches with nothing
// to read but the plan, 2 finding rows and joining sums; the up-projections' 25 MB arrive at 5.3 TB/s, the down-projections' 12 take 4 us,
// h and the plan having come from other units first.
#include "expert_launches.h"
#include "few_rows.h"

#include <type_traits>

namespace mxfp8 {

constexpr int kChunk = 64;      // tokens
constexpr int kUpWaves = 4, kUpThreads = 64 * kUpWaves;  // of a workgroup of the first kernel
constexpr int kMostSlots = 32;  // of a token: 2048 entries of a chunk
constexpr int kMostParts = 256;  // workgroups that share columns of the output, in all
constexpr int64_t kMostLayerWorkgroups = (int64_t(1) << 23) - 1;  // work-items of a launch are numbered in 32 bits

struct LayerRoutes {
    const void *experts;
    const float *weights;
    bool index64;
    int tokens, slots, groups;
    // expert of entry i, -1 for none
    __device__ __forceinline__ int expert(int64_t i) const
    {
        const int64_t e = index64 ? static_cast<const int64_t *>(experts)[i] : (int64_t)static_cast<const int32_t *>(experts)[i];
        return e >= 0 && e < groups ? (int)e : -1;
    }
    __device__ __host__ __forceinline__ int chunk_tokens(int chunk) const
    {
        const int left = tokens - chunk * kChunk;
        return left < kChunk ? left : kChunk;
    }
};

// Plan of a chunk: number of segments of up to `rows` rows, segments {expert, first place << 8 | rows}, entries of the chunk by place
struct LayerPlan {
    int32_t *at;
    int entries;  // at most
    int rows;
    __host__ __device__ static int64_t words(int64_t entries) { return (4 + 3 * entries + 3) / 4 * 4; }
    __device__ __forceinline__ int32_t *segments() const { return at + 4; }
    __device__ __forceinline__ int32_t *places() const { return at + 4 + 2 * entries; }
};

// A token's first entry for an expert stands for all of them. Chunks are walked over in groups of whole tokens.
__device__ __forceinline__ uint64_t lanes_of_token(int lane, int slots)
{
    const int first = lane / slots * slots;
    return (slots == 64 ? ~(uint64_t)0 : ((uint64_t)1 << slots) - 1) << first;
}

// By a workgroup of the first kernel. `lds`: the choices (a token's later ones of the same expert as -1), the experts' rows and where they begin.
__device__ void write_plan(const LayerRoutes &routes, int chunk, const LayerPlan &plan, uint32_t *arrived, uint8_t *lds)
{
    const int tid = threadIdx.x, n = routes.chunk_tokens(chunk) * routes.slots;
    const int64_t base = (int64_t)chunk * kChunk * routes.slots;
    int32_t *const ids = reinterpret_cast<int32_t *>(lds);
    uint32_t *const counts = reinterpret_cast<uint32_t *>(lds) + kChunk * kMostSlots, *const places = counts + routes.groups;
    for (int i = tid; i < n; i += kUpThreads)
        ids[i] = routes.expert(base + i);
    for (int e = tid; e < routes.groups; e += kUpThreads)
        counts[e] = 0;
    static_assert(kMostParts <= kUpThreads, "one count a thread");
    if (chunk == 0 && tid < kMostParts)
        arrived[tid] = 0;
    __syncthreads();
    for (int i0 = 0; i0 < n; i0 += kUpThreads) {
        const int i = i0 + tid;
        bool again = false;
        if (i < n)
            for (int j = i / routes.slots * routes.slots; j < i; ++j)
                again = again || ids[j] == ids[i];
        __syncthreads();
        if (i < n && again)
            ids[i] = -1;  // (what later ones of the token are compared with is the first one, which stays)
        __syncthreads();
    }
    for (int i = tid; i < n; i += kUpThreads)
        if (ids[i] >= 0)
            atomicAdd(&counts[ids[i]], 1u);
    __syncthreads();
    if (tid < 64) {  // places and segments of the experts before each: 64 at a time
        uint32_t place = 0, segment = 0;
        for (int e0 = 0; e0 < routes.groups; e0 += 64) {
            const int e = e0 + tid;
            const uint32_t rows = e < routes.groups ? counts[e] : 0, segments = (rows + plan.rows - 1) / plan.rows;
            uint32_t p = rows, s = segments;
            for (int d = 1; d < 64; d *= 2) {
                const uint32_t lp = (uint32_t)__shfl((int)p, max(tid - d, 0), 64), ls = (uint32_t)__shfl((int)s, max(tid - d, 0), 64);
                p += tid >= d ? lp : 0, s += tid >= d ? ls : 0;
            }
            const uint32_t first = place + p - rows, seg = segment + s - segments;
            if (e < routes.groups)
                places[e] = first;
            for (uint32_t k = 0; k * plan.rows < rows; ++k) {
                plan.segments()[2 * (seg + k)] = e;
                plan.segments()[2 * (seg + k) + 1] = (int32_t)((first + k * plan.rows) << 8 | min(rows - k * plan.rows, (uint32_t)plan.rows));
            }
            place += (uint32_t)__shfl((int)p, 63, 64);
            segment += (uint32_t)__shfl((int)s, 63, 64);
        }
        if (tid == 0)
            plan.at[0] = (int32_t)segment;
    }
    __syncthreads();
    for (int i = tid; i < n; i += kUpThreads)
        if (ids[i] >= 0) {
            uint32_t at = places[ids[i]];
            for (int j = 0; j < i; ++j)
                at += ids[j] == ids[i];
            plan.places()[at] = i;
        }
}

struct LayerWeights {
    FewWeights w;  // of the first expert
    int64_t q_bytes, s_bytes;
    __device__ __forceinline__ FewWeights of(int e) const { return {w.q + e * q_bytes, w.s + e * s_bytes, w.ld, w.N, w.K, w.tiled}; }
};

// WK wavefronts along K, the others along `inter`
template <class Cfg, int WK>
__global__ __launch_bounds__(kUpThreads) void layer_up_kernel(const uint8_t *__restrict__ x, int64_t ldx_bytes, LayerRoutes routes, LayerWeights weights,
                                                               uint32_t blocks_n, uint32_t makers, bool by_entry, uint8_t *__restrict__ h, int planes,
                                                               int32_t *__restrict__ plans, int plan_entries, int plan_rows, uint32_t *__restrict__ arrived)
{
    static_assert(Cfg::NT == 2 && Cfg::MT == 1, "a tile of gates, a tile of the others");
    constexpr int D = Cfg::DEPTH, WN = kUpWaves / WK;
    MXFP8_DYNAMIC_LDS(lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = wave % WK, wn = wave / WK;
    const uint32_t per_chunk = makers * blocks_n + 1;
    const int chunk = (int)(blockIdx.x / per_chunk);
    const uint32_t job = blockIdx.x % per_chunk;
    if (job == 0) {
        write_plan(routes, chunk, {plans + chunk * LayerPlan::words(plan_entries), plan_entries, plan_rows}, arrived, lds);
        return;
    }
    const int maker = (int)((job - 1) / blocks_n), inter = weights.w.N / 2;
    const int n = routes.chunk_tokens(chunk) * routes.slots;
    const int64_t base = (int64_t)chunk * kChunk * routes.slots;
    if (by_entry && maker >= n)
        return;

    // ---- the expert's rows, each wavefront for itself: entries of the chunk and weights
    int32_t *const row_entry = reinterpret_cast<int32_t *>(lds + kUpWaves * Cfg::RING) + wave * 2 * kChunk;
    float *const row_weight = reinterpret_cast<float *>(row_entry + kChunk);
    int rows = 0, expert = by_entry ? -1 : maker;
    const int step = 64 / routes.slots * routes.slots;
    if (by_entry && maker >= step)  // (otherwise it is among the first that are read)
        expert = __builtin_amdgcn_readfirstlane(routes.expert(base + maker));
    for (int i0 = 0; i0 < n; i0 += step) {
        const int i = i0 + lane;
        const bool given = lane < step && i < n;
        const int e = given ? routes.expert(base + i) : -1;
        const float weight = given ? routes.weights[base + i] : 0.0f;
        if (by_entry && i0 == 0 && maker < step)
            expert = __builtin_amdgcn_readlane(e, maker);
        if (expert < 0)
            return;
        const uint64_t chosen = __ballot(e == expert);
        if (by_entry && chosen && rows == 0 && i0 + (int)__builtin_ctzll(chosen) < maker)
            return;  // an earlier entry's workgroups do it (the same for all wavefronts)
        uint64_t mine = chosen & lanes_of_token(lane, routes.slots);
        const bool leads = e == expert && (int)__builtin_ctzll(mine) == lane;
        float sum = weight;
        mine = leads ? mine & (mine - 1) : 0;
        while (__ballot(mine != 0)) {
            const float other = __uint_as_float((uint32_t)__shfl((int)__float_as_uint(weight), mine ? (int)__builtin_ctzll(mine) : lane, 64));
            sum = mine ? sum + other : sum;
            mine &= mine - 1;
        }
        const uint64_t leaders = __ballot(leads);
        if (leads) {
            const int at = rows + __popcll(leaders & (((uint64_t)1 << lane) - 1));
            row_entry[at] = i;
            row_weight[at] = sum;
        }
        rows += __popcll(leaders);
    }
    if (rows == 0)
        return;
    __builtin_amdgcn_wave_barrier();
    MXFP8_FENCE();

    const FewWeights w = weights.of(expert);
    const int n0 = ((int)((job - 1) % blocks_n) * WN + wn) * 16, tile_n = min(n0, (inter - 1) & ~15);
    FewStream<Cfg> stream;
    stream.init(lds, wave, lane, w.K);
    const int begin = (int)((int64_t)stream.units * wk / WK), end = (int)((int64_t)stream.units * (wk + 1) / WK);
    const float *scales[2];
    int shift[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int at = tile_n + t * inter;
        stream.tile(t, w, at);
        scales[t] = reinterpret_cast<const float *>(w.s) + (int64_t)(at >> 7) * stream.units;
        shift[t] = Cfg::MX ? FewStream<Cfg>::scale_shift(w, min(at + stream.r, w.N - 1), stream.g) : 0;
    }
    for (int first = 0; first < rows; first += Cfg::XR) {
        const int count = min(rows - first, Cfg::XR);
        stream.rows(x, [&](int m) { return (uint32_t)(((int)base + row_entry[first + min(m, count - 1)]) / routes.slots) * (uint32_t)ldx_bytes; });
        typename FewStream<Cfg>::Sums sums_k = {};
        auto &acc = sums_k[0];
        for (int u = begin; u < min(begin + D, end); ++u)
            stream.issue(u, (u - begin) % D, w.tiled);
        for (int u = begin; u < end; ++u) {
            const int slot = (u - begin) % D;
            float scale[2] = {1.0f, 1.0f};
            if constexpr (!Cfg::MX)
                scale[0] = scalar_load(scales[0] + u), scale[1] = scalar_load(scales[1] + u);
            stream.wait(end - 1 - u);
            MXFP8_FENCE();
            stream.read(u, slot, shift);
            if (u + D < end) {
                MXFP8_FENCE();
                MXFP8_WAIT_VMCNT_AND_LDS(63);  // (the slot's reads have returned)
                MXFP8_FENCE();
                stream.issue(u + D, slot, w.tiled);
            }
            stream.multiply(sums_k, scale);
        }
        if constexpr (WK > 1) {
            static_assert(2 * 1024 <= Cfg::RING, "the sums take the ring's place");
            MXFP8_FENCE();
            __syncthreads();
            v4f *const sums = reinterpret_cast<v4f *>(lds);
            sums[(wave * 2) * 64 + lane] = acc[0][0];
            sums[(wave * 2 + 1) * 64 + lane] = acc[1][0];
            __syncthreads();
            if (wk == 0)
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int v = 1; v < WK; ++v)
                        acc[t][0] += sums[((wave + v) * 2 + t) * 64 + lane];
            __syncthreads();  // the next rows' units go where the sums are
        }
        const int at = n0 + 4 * stream.g;
        if (wk == 0 && stream.r < count && at < inter) {
            const int entry = row_entry[first + stream.r];
            const float weight = row_weight[first + stream.r];
            uint32_t part[3][2] = {};
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float gate = acc[0][0][v];
                float rest = weight * (gate / (1.0f + expf(-gate)) * acc[1][0][v]);
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    const __bf16 high = (__bf16)rest;
                    part[p][v / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, high) << (16 * (v & 1));
                    rest -= (float)high;
                    rest = rest - rest == 0.0f ? rest : 0.0f;  // an infinity leaves none
                }
            }
            uint8_t *const to = h + (base + entry) * planes * inter * 2 + at * 2;
#pragma unroll
            for (int p = 0; p < 3; ++p)
                if (p < planes)
                    *reinterpret_cast<uint2 *>(to + (int64_t)p * inter * 2) = make_uint2(part[p][0], part[p][1]);
        }
    }
}

template <class Cfg>
__global__ __launch_bounds__(kFewThreads) void layer_down_kernel(const uint8_t *__restrict__ h, const int32_t *__restrict__ plans, int plan_entries,
                                                                 LayerRoutes routes, LayerWeights weights, uint32_t blocks_n, int parts, int chunk_rows,
                                                                 uint32_t *__restrict__ arrived, float *__restrict__ part_sums,
                                                                 uint8_t *__restrict__ out, bool out_bf16, int64_t ld_out)
{
    static_assert(Cfg::NT == 1 && Cfg::MT == 1 && Cfg::PLANES >= 2, "segments of one tile of h's rows");
    constexpr int D = Cfg::DEPTH;
    MXFP8_DYNAMIC_LDS(lds);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // (parts > 1: of the only chunk)
    const int block = (int)(blockIdx.x % blocks_n), chunk = parts > 1 ? 0 : (int)(blockIdx.x / blocks_n), part = parts > 1 ? (int)(blockIdx.x / blocks_n) : 0;
    const int n0 = block * 16, tokens = routes.chunk_tokens(chunk), inter = weights.w.K;
    const int64_t base = (int64_t)chunk * kChunk * routes.slots;
    float *const sums = reinterpret_cast<float *>(lds + kFewWaves * Cfg::RING);  // [wavefront][token][16]
    int32_t *const plan_lds = reinterpret_cast<int32_t *>(sums + kFewWaves * chunk_rows * 16);
    const int32_t *const from = plans + chunk * LayerPlan::words(plan_entries);
    for (int i = tid; i < 4 + 3 * plan_entries; i += kFewThreads)  // (all of it: how much there is would have to be waited for)
        plan_lds[i] = from[i];
    for (int i = tid; i < kFewWaves * chunk_rows * 16; i += kFewThreads)
        sums[i] = 0.0f;
    __syncthreads();
    const LayerPlan plan = {plan_lds, plan_entries, 0};
    const int segments = __builtin_amdgcn_readfirstlane(plan_lds[0]);

    FewStream<Cfg> stream;
    stream.init(lds, wave, lane, inter);
    const int units = max(stream.units, 1);  // (none: there are no segments)
    const int64_t all = (int64_t)segments * units;
    const int mine = part * kFewWaves + wave, sharers = parts * kFewWaves;
    const int begin = (int)(all * mine / sharers), end = (int)(all * (mine + 1) / sharers);
    // what is being requested, and what is being multiplied: a segment and a unit of it
    int seg_in = begin / units, u_in = begin % units, seg = seg_in, u = u_in;
    const int n = min(n0, weights.w.N - 1);
    auto open = [&](int s) __attribute__((always_inline)) {
        const int expert = __builtin_amdgcn_readfirstlane(plan.segments()[2 * s]), rows = __builtin_amdgcn_readfirstlane(plan.segments()[2 * s + 1]);
        const int first = rows >> 8, count = rows & 255;
        stream.tile(0, weights.of(expert), n);
        stream.rows(h + base * Cfg::PLANES * inter * 2, [&](int m) {
            return ((uint32_t)plan.places()[first + min(m % Cfg::XR, count - 1)] * Cfg::PLANES + (uint32_t)(m / Cfg::XR)) * (uint32_t)inter * 2;
        });
    };
    auto request = [&](int slot) __attribute__((always_inline)) {
        stream.issue(u_in, slot, weights.w.tiled);
        if (++u_in == units) {
            u_in = 0;
            ++seg_in;
        }
    };
    int shift[1] = {Cfg::MX ? FewStream<Cfg>::scale_shift(weights.w, min(n + stream.r, weights.w.N - 1), stream.g) : 0};
    typename FewStream<Cfg>::Sums acc = {};
    if (begin < end)
        open(seg_in);
    for (int k = begin; k < min(begin + D, end); ++k) {
        request((k - begin) % D);
        if (u_in == 0 && k + 1 < end)
            open(seg_in);
    }
    for (int k = begin; k < end; ++k) {
        const int slot = (k - begin) % D;
        const int row = __builtin_amdgcn_readfirstlane(plan.segments()[2 * seg + 1]);
        float scale[1] = {1.0f};
        if constexpr (!Cfg::MX)
            scale[0] = scalar_load(reinterpret_cast<const float *>(weights.w.s + __builtin_amdgcn_readfirstlane(plan.segments()[2 * seg]) * weights.s_bytes) +
                                   (int64_t)(n >> 7) * units + u);
        stream.wait(end - 1 - k);
        MXFP8_FENCE();
        stream.read(u, slot, shift);
        if (k + D < end) {
            MXFP8_FENCE();
            MXFP8_WAIT_VMCNT_AND_LDS(63);  // (the slot's reads have returned)
            MXFP8_FENCE();
            request(slot);
            if (u_in == 0 && k + D + 1 < end)
                open(seg_in);
        }
        stream.multiply(acc, scale);
        if (++u == units || k + 1 == end) {  // this wavefront's part of the segment
            if (stream.r < (row & 255)) {
                const int token = plan.places()[(row >> 8) + stream.r] / routes.slots;
                v4f *const to = reinterpret_cast<v4f *>(sums + (wave * chunk_rows + token) * 16 + 4 * stream.g);
                *to += FewStream<Cfg>::total(acc, 0, 0);
            }
#pragma unroll
            for (int p = 0; p < Cfg::PLANES; ++p)
                acc[p][0][0] = v4f{0.f, 0.f, 0.f, 0.f};
            u = 0;
            ++seg;
        }
    }
    MXFP8_FENCE();
    __syncthreads();
    const int given = tokens * 16;
    auto of_wavefronts = [&](int i) __attribute__((always_inline)) {
        float sum = sums[i];
#pragma unroll
        for (int v = 1; v < kFewWaves; ++v)
            sum += sums[v * chunk_rows * 16 + i];
        return sum;
    };
    auto store = [&](int i, float sum) __attribute__((always_inline)) {
        const int column = n0 + (i & 15);
        const int64_t to = ((int64_t)chunk * kChunk + (i >> 4)) * ld_out + column;
        if (column < weights.w.N) {
            if (out_bf16)
                reinterpret_cast<__bf16 *>(out)[to] = (__bf16)sum;
            else
                reinterpret_cast<float *>(out)[to] = sum;
        }
    };
    if (parts == 1) {
        for (int i = tid; i < given; i += kFewThreads)
            store(i, of_wavefronts(i));
        return;
    }
    // The workgroup that arrives last adds up what all of them have left, in the order of the parts. Sums are written and read past the
    // caches that are not shared (device-wide accesses), and each wavefront waits for its own to have been written before the workgroup
    // counts itself: nothing else has to be made visible, and a fence that writes a whole L2 back takes 20 us here.
    const int64_t stride = (int64_t)blocks_n * chunk_rows * 16;
    float *const place = part_sums + (int64_t)block * chunk_rows * 16;
    for (int i = tid; i < given; i += kFewThreads)
        __hip_atomic_store(place + part * stride + i, of_wavefronts(i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    MXFP8_FENCE();
    MXFP8_WAIT_VMCNT_AND_LDS(0);
    __syncthreads();
    uint32_t *const order = reinterpret_cast<uint32_t *>(lds);
    if (tid == 0)
        *order = atomicAdd(&arrived[block], 1u);
    __syncthreads();
    if (*order != (uint32_t)parts - 1)
        return;
    MXFP8_FENCE();
    for (int i = tid; i < given; i += kFewThreads) {
        float sum = __hip_atomic_load(place + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        for (int p = 1; p < parts; ++p)
            sum += __hip_atomic_load(place + p * stride + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        store(i, sum);
    }
}

static int64_t layer_h_bytes(int64_t tokens, int slots, int64_t inter) { return (tokens * slots * inter * 6 + 15) / 16 * 16; }  // three planes
static int64_t layer_chunk_rows(int64_t tokens) { return tokens < kChunk ? tokens : kChunk; }
static int64_t layer_plan_bytes(int64_t tokens, int slots)
{
    return (tokens + kChunk - 1) / kChunk * LayerPlan::words(layer_chunk_rows(tokens) * slots) * 4;
}
int64_t expert_layer_workspace(int64_t tokens, int slots, int64_t inter)
{
    return layer_h_bytes(tokens, slots, inter) + layer_plan_bytes(tokens, slots) + kMostParts * 4 + kMostParts * layer_chunk_rows(tokens) * 64;
}

template <class Kernel> static hipError_t allow_lds(Kernel kern, int bytes)
{
    return hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

struct LayerCall {
    const uint8_t *x;
    int64_t ldx;
    LayerRoutes routes;
    LayerWeights up, down;
    uint8_t *out;
    bool out_bf16;
    int64_t ld_out;
    uint8_t *h;
    int32_t *plans;
    uint32_t *arrived;
    float *part_sums;
    int entries;  // of a chunk
    int64_t chunks;
    hipStream_t stream;
};

template <class Cfg> static hipError_t launch_up(const LayerCall &c, int plan_rows)
{
    const bool by_entry = c.entries <= c.routes.groups;
    const int64_t inter = c.down.w.K, makers = by_entry ? c.entries : c.routes.groups, tiles = (inter + 15) / 16 * makers * c.chunks;
    const int64_t units = (c.up.w.K + 127) / 128;
    int wk = 1;
    while (wk < kUpWaves && units >= 2 * wk && tiles * wk * 2 <= 8192)
        wk *= 2;
    const int64_t blocks_n = (inter + 16 * (kUpWaves / wk) - 1) / (16 * (kUpWaves / wk)), grid = (makers * blocks_n + 1) * c.chunks;
    if (grid > kMostLayerWorkgroups)
        return hipErrorInvalidConfiguration;
    // rings and the rows of each wavefront, or the choices and counts that the plan is made of
    const int list_bytes = kUpWaves * (Cfg::RING + 2 * kChunk * 4), plan_bytes = (kChunk * kMostSlots + 2 * c.routes.groups) * 4;
    const int bytes = list_bytes > plan_bytes ? list_bytes : plan_bytes;
    auto kern = wk == 1 ? layer_up_kernel<Cfg, 1> : wk == 2 ? layer_up_kernel<Cfg, 2> : layer_up_kernel<Cfg, 4>;
    const hipError_t e = allow_lds(kern, bytes);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(kUpThreads), bytes, c.stream, c.x, c.ldx * 2, c.routes, c.up, (uint32_t)blocks_n, (uint32_t)makers,
                       by_entry, c.h, c.out_bf16 ? 2 : 3, c.plans, c.entries, plan_rows, c.arrived);
    return hipGetLastError();
}

template <class Cfg> static hipError_t launch_down(const LayerCall &c)
{
    const int64_t blocks_n = (c.down.w.N + 15) / 16, chunk_rows = layer_chunk_rows(c.routes.tokens);
    // units of a wavefront, if every choice is another expert's; parts as long as they leave it some
    const int64_t all = min((int64_t)c.entries, (int64_t)c.routes.groups) * ((c.down.w.K + 127) / 128) / kFewWaves;
    int parts = 1;
    while (c.chunks == 1 && blocks_n * parts * 2 <= kMostParts && all >= 8 * parts)
        parts *= 2;
    const int bytes = (int)(kFewWaves * (Cfg::RING + chunk_rows * 64) + LayerPlan::words(c.entries) * 4);
    auto kern = layer_down_kernel<Cfg>;
    const hipError_t e = allow_lds(kern, bytes);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(blocks_n * parts * c.chunks)), dim3(kFewThreads), bytes, c.stream, c.h, c.plans, c.entries, c.routes, c.down,
                       (uint32_t)blocks_n, parts, (int)chunk_rows, c.arrived, c.part_sums, c.out, c.out_bf16, c.ld_out);
    return hipGetLastError();
}

template <int FMT> static hipError_t launch_layer(const LayerCall &c)
{
    if ((c.down.w.N + 15) / 16 * c.chunks > kMostLayerWorkgroups)
        return hipErrorInvalidConfiguration;
    // Rows that an expert is made ready for: what it has in the mean is known, and the ones that are chosen have more than that.
    const int64_t tokens = c.routes.tokens, rows = tokens == 1 ? 1 : min(tokens, (int64_t)c.entries * 3 / 2 / max(c.routes.groups, 1) + 1);
    constexpr bool FP4 = FMT == kWeightsFp4;
    auto up = tokens == 1 ? launch_up<FewCfg<FMT, 1, 2, 1, 2>>
              : rows <= 4 ? launch_up<FewCfg<FMT, 4, 2, 1, 2>>
              : rows <= 8 ? launch_up<FewCfg<FMT, 8, 2, 1, 2>>
                          : launch_up<FewCfg<FMT, 16, 2, 1, 2>>;
    // (four units of MXFP4 do not fit LDS beside the plan of more entries; nor do eight rows in three planes)
    const int plan_rows = tokens == 1 ? 1 : !c.out_bf16 || (rows <= 3 && c.entries <= 1536) ? 4 : 8;
    auto down = c.out_bf16 ? plan_rows == 1   ? launch_down<FewCfg<FMT, 1, 1, 2, 3>>
                             : plan_rows == 4 ? launch_down<FewCfg<FMT, 4, 1, 2, FP4 ? 4 : 3>>
                                              : launch_down<FewCfg<FMT, 8, 1, 2, 2>>
                : plan_rows == 1 ? launch_down<FewCfg<FMT, 1, 1, 3, 3>>
                                 : launch_down<FewCfg<FMT, 4, 1, 3, 2>>;
    const hipError_t e = up(c, plan_rows);
    return e == hipSuccess ? down(c) : e;
}

hipError_t launch_expert_layer(const void *x, int64_t tokens, int64_t hidden, int64_t ldx, const void *experts, bool index64, int slots,
                               const float *weights, int format, const uint8_t *up_q, const void *up_s, int64_t up_s_bytes, const uint8_t *down_q,
                               const void *down_s, int64_t down_s_bytes, int groups, int64_t inter, void *out, bool out_bf16, int64_t ld_out,
                               void *workspace, bool tiled_scales, hipStream_t stream)
{
    const LayerRoutes routes = {experts, weights, index64, (int)tokens, slots, groups};
    auto matrices = [&](const uint8_t *q, const void *s, int64_t s_bytes, int64_t rows, int64_t cols) {
        const int64_t ld = format == kWeightsFp4 ? cols / 2 : cols;
        return LayerWeights{{q, static_cast<const uint8_t *>(s), ld, (int)rows, (int)cols, tiled_scales}, rows * ld, s_bytes};
    };
    const LayerWeights up = matrices(up_q, up_s, up_s_bytes, 2 * inter, hidden), down = matrices(down_q, down_s, down_s_bytes, hidden, inter);
    uint8_t *const plans = static_cast<uint8_t *>(workspace) + layer_h_bytes(tokens, slots, inter), *const arrived = plans + layer_plan_bytes(tokens, slots);
    const LayerCall call = {static_cast<const uint8_t *>(x), ldx, routes, up, down, static_cast<uint8_t *>(out), out_bf16, ld_out, static_cast<uint8_t *>(workspace),
                            reinterpret_cast<int32_t *>(plans), reinterpret_cast<uint32_t *>(arrived), reinterpret_cast<float *>(arrived + kMostParts * 4),
                            (int)layer_chunk_rows(tokens) * slots, (tokens + kChunk - 1) / kChunk, stream};
    return format == kWeightsFp4 ? launch_layer<kWeightsFp4>(call) : format == kWeightsFp8 ? launch_layer<kWeightsFp8>(call) : launch_layer<kWeightsB128>(call);
}

}  // namespace mxfp8
