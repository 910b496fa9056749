// Entries (tokens times slots) sorted by expert: a stable counting sort with padded ends (include/mxfp8_experts.h).
//
// position(i) = begin(e_i) + number of earlier entries of the same expert, begin = prefix sum of the padded counts. Each workgroup
// owns a run of consecutive entries and needs, besides the counts of all experts, those of the entries before its own. Up to
// kOneLaunch entries every workgroup counts them itself, from all entries: one launch and no workspace. Beyond, a first launch
// counts each run into the workspace. There are no atomics on global memory and no waits between workgroups; counts are whole numbers, so
// the order of the LDS atomics does not matter.
//   What bounds it is latency: launches, the counts, three barriers for 1024 entries. In a captured graph, where an empty kernel takes 2.2
// us: 48 entries of 64 experts 4.8 us, 131072 of 128 experts 9.1, 524288 of 256 16.6 (their bytes alone, 6.4 MB, would take 1.2); launched one
// after the other, where an empty kernel takes 3.8, the first two take 4.3 and 8.6.
#include "expert_launches.h"
#include "mxfp8_device.h"

namespace mxfp8 {

constexpr int64_t kOneLaunch = 8192;  // 8192 entries of 16 | 256 experts: 6.3 | 7.1 us in one launch, 6.9 | 8.2 in two; 16384: 8.0 | 8.5, 7.0 | 8.8
constexpr int kSortThreads = 1024;
constexpr unsigned kFill = 2048;  // rows that a workgroup fills
constexpr int kRuns = 256;  // at most, where there are two launches: every workgroup reads the counts of all runs

// entries of a run where there are two launches
static int64_t run_of(int64_t entries)
{
    return ((entries + kRuns - 1) / kRuns + kSortThreads - 1) / kSortThreads * kSortThreads;
}

// expert of entry i, `groups` for none
template <class ID> __device__ __forceinline__ int expert_of(const ID *__restrict__ experts, int i, int groups)
{
    const ID e = experts[i];
    return e >= 0 && e < (ID)groups ? (int)e : groups;
}

// counts[run][expert]
template <class ID>
__global__ __launch_bounds__(kSortThreads) void expert_count_kernel(const ID *__restrict__ experts, int entries, int groups, int run,
                                                                    uint32_t *__restrict__ counts)
{
    MXFP8_DYNAMIC_LDS(lds);
    uint32_t *const count = reinterpret_cast<uint32_t *>(lds);
    const int tid = threadIdx.x, n = blockDim.x;
    for (int e = tid; e < groups; e += n)
        count[e] = 0;
    __syncthreads();
    const int first = blockIdx.x * run, last = min(first + run, entries);
    for (int i = first + tid; i < last; i += n) {
        const int e = expert_of(experts, i, groups);
        if (e < groups)
            atomicAdd(count + e, 1u);
    }
    __syncthreads();
    for (int e = tid; e < groups; e += n)
        counts[(int64_t)blockIdx.x * groups + e] = count[e];
}

// Workgroup b places the entries [b * run, (b + 1) * run). counts == nullptr: it counts all entries itself.
// LDS: groups words each of next (the row of the expert's next entry), begin and total, 16 words of sums, and a byte for each wavefront
// and expert: how many of the wavefront's entries are the expert's.
template <class ID>
__global__ __launch_bounds__(kSortThreads) void expert_sort_kernel(const ID *__restrict__ experts, int entries, int groups, int align, int rows, int run,
                                                           int32_t *__restrict__ positions, int32_t *__restrict__ sources,
                                                           int32_t *__restrict__ group_ends, const uint32_t *__restrict__ counts)
{
    MXFP8_DYNAMIC_LDS(lds);
    uint32_t *const next = reinterpret_cast<uint32_t *>(lds), *const begin = next + groups, *const total = begin + groups, *const sums = total + groups;
    uint8_t *const own = reinterpret_cast<uint8_t *>(sums + kSortThreads / 64);
    const int tid = threadIdx.x, n = blockDim.x, lane = tid & 63, wave = tid >> 6, waves = n >> 6;
    const int first = blockIdx.x * run, last = min(first + run, entries);

    // ---- counts: of all entries, and of those before this workgroup's
    for (int e = tid; e < groups; e += n)
        next[e] = total[e] = 0;
    for (int i = tid; i < waves * groups; i += n)
        own[i] = 0;
    __syncthreads();
    if (counts == nullptr) {
        for (int i = tid; groups > 0 && i < entries; i += n) {  // more than kOneLaunch entries only come here without experts
            const int e = expert_of(experts, i, groups);
            if (e < groups) {
                atomicAdd(total + e, 1u);
                if (i < first)
                    atomicAdd(next + e, 1u);
            }
        }
    } else {
        const int runs = gridDim.x, side_by_side = max(n / max(groups, 1), 1);  // so many work-items share an expert
        for (int e = tid % max(groups, 1), b0 = tid / max(groups, 1); b0 < side_by_side && e < groups; e += n) {
            uint32_t all = 0, before = 0;
            for (int b1 = b0; b1 < runs; b1 += 16 * side_by_side) {  // sixteen loads on their way at a time
                uint32_t c[16];
#pragma unroll
                for (int k = 0; k < 16; ++k)
                    c[k] = counts[(int64_t)min(b1 + k * side_by_side, runs - 1) * groups + e];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const int b = b1 + k * side_by_side;
                    all += b < runs ? c[k] : 0;
                    before += b < min(runs, (int)blockIdx.x) ? c[k] : 0;
                }
            }
            atomicAdd(total + e, all);
            atomicAdd(next + e, before);
        }
    }
    __syncthreads();

    // ---- padded ends: each work-item adds up its share of the experts, then the shares are summed over lanes and wavefronts
    const int share = (groups + n - 1) / n;
    const uint32_t pad = (uint32_t)align - 1;
    uint32_t mine = 0;
    for (int e = tid * share; e < min((tid + 1) * share, groups); ++e)
        mine += (total[e] + pad) & ~pad;
    uint32_t upto = mine;  // inclusive over the lanes
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = (uint32_t)__shfl((int)upto, lane >= d ? lane - d : lane, 64);
        upto += lane >= d ? o : 0;
    }
    if (lane == 63)
        sums[wave] = upto;
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (int w = 0; w < waves; ++w) {
        before += w < wave ? sums[w] : 0;
        all += sums[w];
    }
    uint32_t at = before + upto - mine;
    for (int e = tid * share; e < min((tid + 1) * share, groups); ++e) {
        begin[e] = at;
        next[e] += at;
        at += (total[e] + pad) & ~pad;
        if (blockIdx.x == 0)
            group_ends[e] = (int32_t)at;
    }
    __syncthreads();

    // ---- rows of the padding, the experts dealt out to the wavefronts of all workgroups, and rows behind the last expert
    for (int e = blockIdx.x * waves + wave; e < groups; e += gridDim.x * waves) {
        const uint32_t end = begin[e] + ((total[e] + pad) & ~pad);
        for (uint32_t r = begin[e] + total[e] + lane; r < end; r += 64)
            sources[r] = -1;
    }
    for (int64_t r = (int64_t)all + blockIdx.x * n + tid; r < rows; r += (int64_t)gridDim.x * n)
        sources[r] = -1;

    // ---- places: a work-item takes an entry. Lanes of the same expert find each other by the bits of its number; the first of them
    // says how many they are and adds up what the wavefronts before it have.
    const int bits = 32 - __builtin_clz((unsigned)groups | 1u);
    for (int i0 = first; i0 < last; i0 += n) {
        const int i = i0 + tid;
        const int e = i < last ? expert_of(experts, i, groups) : groups;
        uint64_t same = ~(uint64_t)0;
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot((e >> b) & 1);
            same &= ((e >> b) & 1) ? set : ~set;
        }
        const int rank = __popcll(same & (((uint64_t)1 << lane) - 1)), many = __popcll(same);
        const bool leads = rank == 0 && e < groups;
        if (leads)
            own[wave * groups + e] = (uint8_t)many;
        __syncthreads();
        uint32_t base = 0;
        if (leads) {
            base = next[e];
            for (int w = 0; w < wave; ++w)
                base += own[w * groups + e];
        }
        base = (uint32_t)__shfl((int)base, (int)__builtin_ctzll(same), 64);
        if (i < last) {
            const int row = e < groups ? (int)base + rank : -1;
            positions[i] = row;
            if (row >= 0)
                sources[row] = i;
        }
        if (i0 + n < last) {
            __syncthreads();
            if (leads) {
                own[wave * groups + e] = 0;
                atomicAdd(next + e, (uint32_t)many);
            }
            __syncthreads();
        }
    }
}

int64_t expert_sort_workspace(int64_t entries, int groups)
{
    return entries > kOneLaunch ? (entries + run_of(entries) - 1) / run_of(entries) * groups * 4 : 0;
}

template <class ID>
static hipError_t launch_expert_sort_t(const ID *experts, int entries, int groups, int align, int rows, int32_t *positions, int32_t *sources,
                                       int32_t *group_ends, uint32_t *counts, hipStream_t stream)
{
    const bool two = entries > kOneLaunch && groups > 0;
    const int threads = entries <= 256 ? 256 : kSortThreads, run = two ? (int)run_of(entries) : threads;
    // One launch: where the padding has many more rows than there are entries, further workgroups (they count too) help to fill it.
    // (512 entries of 256 experts, 33152 rows: 7.5 us with one workgroup.)
    const unsigned runs = entries > 0 ? (unsigned)((entries + run - 1) / run) : 1u;
    const unsigned workgroups = two ? runs : max(runs, min(((unsigned)rows + kFill - 1) / kFill, 64u));
    const size_t lds = ((size_t)groups * 3 + kSortThreads / 64) * 4 + (size_t)(threads / 64) * groups;  // 112 KB for 4096 experts
    hipError_t e = hipSuccess;
    if (lds > 64 * 1024)
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(expert_sort_kernel<ID>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess)
        return e;
    if (two) {
        hipLaunchKernelGGL((expert_count_kernel<ID>), dim3(workgroups), dim3(kSortThreads), (size_t)groups * 4, stream, experts, entries, groups, run,
                           counts);
        e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    hipLaunchKernelGGL((expert_sort_kernel<ID>), dim3(workgroups), dim3(threads), lds, stream, experts, entries, groups, align, rows, run, positions,
                       sources, group_ends, two ? counts : nullptr);
    return hipGetLastError();
}

hipError_t launch_expert_sort(const void *experts, bool index64, int64_t entries, int groups, int align, int64_t rows, int32_t *positions,
                              int32_t *sources, int32_t *group_ends, uint32_t *workspace, hipStream_t stream)
{
    return index64 ? launch_expert_sort_t(static_cast<const int64_t *>(experts), (int)entries, groups, align, (int)rows, positions, sources,
                                          group_ends, workspace, stream)
                   : launch_expert_sort_t(static_cast<const int32_t *>(experts), (int)entries, groups, align, (int)rows, positions, sources,
                                          group_ends, workspace, stream);
}

}  // namespace mxfp8
