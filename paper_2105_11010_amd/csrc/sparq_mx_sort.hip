// The router's choices sorted by expert (include/sparq_mx_experts.h).
#include "sparq_mx_experts.h"

namespace sparq {
namespace mx {

// A counting sort that keeps the order of equal keys.  A wavefront has a range of slots: it counts them by expert in LDS, and once the counts of
// all ranges before its own are known, for each expert, it takes 64 slots at a time; a slot's rank among the lanes with the same expert is the number of
// such lanes below, found by one ballot a bit of the expert's number.  Slots refused are those of one expert more, the last.
struct SortParams {
    const int32_t* expert;
    int32_t *offsets, *place, *order;
    int32_t* counts;             // [workgroups][experts + 1], of more workgroups than one
    int32_t slots, experts, range, ranges;       // slots of a wavefront (whole 64s), and all wavefronts
};

template <int WAVES>
__device__ __forceinline__ void count_own(const SortParams& p, int32_t* mine, int first, int last) {
    const int lane = threadIdx.x & 63;
    for (int s = first + lane; s < last; s += 64) {
        const int e = p.expert[s];
        atomicAdd(&mine[(unsigned)e < (unsigned)p.experts ? e : p.experts], 1);
    }
}

// Counts of a workgroup's slots
template <int WAVES>
__global__ __launch_bounds__(WAVES * 64) void sort_count_kernel(const SortParams p) {
    extern __shared__ int32_t counts[];
    const int buckets = p.experts + 1;
    for (int i = threadIdx.x; i < buckets; i += WAVES * 64) counts[i] = 0;
    __syncthreads();
    const int64_t first = (int64_t)(blockIdx.x * WAVES + (threadIdx.x >> 6)) * p.range, last = first + p.range;
    count_own<WAVES>(p, counts, (int)(first < p.slots ? first : p.slots), (int)(last < p.slots ? last : p.slots));
    __syncthreads();
    for (int i = threadIdx.x; i < buckets; i += WAVES * 64) p.counts[(int64_t)blockIdx.x * buckets + i] = counts[i];
}

template <int WAVES, bool MANY>
__global__ __launch_bounds__(WAVES * 64) void sort_kernel(const SortParams p) {
    constexpr int THREADS = WAVES * 64;
    extern __shared__ int32_t lds[];             // [WAVES][buckets] counts, then the wavefronts' next rows; [buckets] all counts; [WAVES] sums
    const int buckets = p.experts + 1, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t *const mine = lds + wave * buckets, *const all = lds + WAVES * buckets, *const sums = all + buckets;
    for (int i = threadIdx.x; i < WAVES * buckets; i += THREADS) lds[i] = 0;
    __syncthreads();
    const int64_t begin = (int64_t)(blockIdx.x * WAVES + wave) * p.range, end = begin + p.range;
    const int first = (int)(begin < p.slots ? begin : p.slots), last = (int)(end < p.slots ? end : p.slots);
    count_own<WAVES>(p, mine, first, last);
    __syncthreads();
    // Counts before each wavefront, and all of them
    for (int e = threadIdx.x; e < buckets; e += THREADS) {
        int before = 0;
        if constexpr (MANY)
            for (int b = 0; b < (int)blockIdx.x; ++b) before += p.counts[(int64_t)b * buckets + e];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int n = lds[w * buckets + e];
            lds[w * buckets + e] = before;
            before += n;
        }
        if constexpr (MANY)
            for (int b = blockIdx.x + 1; b < (int)gridDim.x; ++b) before += p.counts[(int64_t)b * buckets + e];
        all[e] = before;
    }
    __syncthreads();
    // The experts' first rows: sums of the counts below, THREADS experts at a time
    int carried = 0;
    for (int e0 = 0; e0 < buckets; e0 += THREADS) {
        const int e = e0 + (int)threadIdx.x, n = e < buckets ? all[e] : 0;
        int sum = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(sum, d);
            if (lane >= d) sum += v;
        }
        if (lane == 63) sums[wave] = sum;
        __syncthreads();
        int below = carried, total = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) below += sums[w];
            total += sums[w];
        }
        carried += total;
        if (e < buckets) {
            const int row = below + sum - n;
            if (blockIdx.x == 0) p.offsets[e] = row;         // (the refused ones' first row is the number of rows)
#pragma unroll
            for (int w = 0; w < WAVES; ++w) lds[w * buckets + e] += row;
        }
        __syncthreads();
    }
    const int bits = 32 - __builtin_clz(p.experts);
    for (int s0 = first; s0 < last; s0 += 64) {
        const int s = s0 + lane, e = s < last ? p.expert[s] : -1, key = (unsigned)e < (unsigned)p.experts ? e : p.experts;
        uint64_t same = __ballot(s < last);
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot(key >> b & 1);
            same &= key >> b & 1 ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        if (s < last) {
            const int row = mine[key] + rank;
            p.place[s] = key < p.experts ? row : -1;
            if (p.order) p.order[row] = key < p.experts ? s : -1;
        }
        wavefront_lds_fence();
        if (s < last && rank == 0) mine[key] += __popcll(same);
        wavefront_lds_fence();
    }
}

constexpr int kSortWaves = 8;
// One workgroup up to this many slots; more take two launches, the first of which counts.
struct SortPlan {
    int waves, range, blocks;
    size_t bytes;
};
static SortPlan sort_plan(int64_t slots, int experts) {
    SortPlan p = {};
    p.waves = slots <= 128 ? 1 : kSortWaves;
    const int64_t wanted = slots <= 8192 ? p.waves : (slots + 511) / 512;
    const int64_t ranges = wanted < 1024 ? wanted : 1024;
    p.range = (int)round_up((slots + ranges - 1) / ranges, 64);
    p.blocks = slots == 0 ? 1 : (int)((slots + (int64_t)p.range * p.waves - 1) / ((int64_t)p.range * p.waves));
    p.bytes = p.blocks > 1 ? (size_t)round_up((int64_t)p.blocks * (experts + 1) * 4, 256) : 0;
    return p;
}
static bool sort_sizes_ok(int64_t slots, int experts) { return slots >= 0 && experts >= 1; }
static bool sort_countable(int64_t slots, int experts) { return slots <= 1 << 30 && experts <= SPARQ_MX_EXPERTS_MOST; }

}  // namespace mx
}  // namespace sparq

using namespace sparq;
using namespace sparq::mx;

extern "C" size_t sparq_mx_sort_workspace_bytes(int64_t slots, int32_t experts) {
    return sort_sizes_ok(slots, experts) && sort_countable(slots, experts) ? sort_plan(slots, experts).bytes : 0;
}

extern "C" sparq_status sparq_mx_sort(const int32_t* expert, int64_t slots, int32_t experts, int32_t* offsets, int32_t* place, int32_t* order,
                                      void* workspace, size_t workspace_bytes, void* stream) {
    if (!sort_sizes_ok(slots, experts)) return SPARQ_EINVAL;
    if (!offsets || !aligned(offsets, 4) || !aligned(order, 4)) return SPARQ_EINVAL;
    if (slots > 0 && (!expert || !aligned(expert, 4) || !place || !aligned(place, 4))) return SPARQ_EINVAL;
    if (!sort_countable(slots, experts)) return SPARQ_EUNSUPPORTED;
    const SortPlan plan = sort_plan(slots, experts);
    if (plan.bytes && (!workspace || !aligned(workspace, 256))) return SPARQ_EINVAL;
    if (workspace_bytes < plan.bytes) return SPARQ_EWORKSPACE;
    const SortParams p = {expert, offsets, place, order, static_cast<int32_t*>(workspace), (int32_t)slots, experts, plan.range, 0};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int buckets = experts + 1;
    if (plan.waves == 1) {
        sort_kernel<1, false><<<1, 64, (2 * buckets + 1) * 4, s>>>(p);
        return launch_status();
    }
    const int lds_bytes = ((kSortWaves + 1) * buckets + kSortWaves) * 4;
    if (plan.blocks == 1) {
        sort_kernel<kSortWaves, false><<<1, kSortWaves * 64, lds_bytes, s>>>(p);
        return launch_status();
    }
    sort_count_kernel<kSortWaves><<<plan.blocks, kSortWaves * 64, buckets * 4, s>>>(p);
    const sparq_status counted = launch_status();
    if (counted != SPARQ_OK) return counted;
    sort_kernel<kSortWaves, true><<<plan.blocks, kSortWaves * 64, lds_bytes, s>>>(p);
    return launch_status();
}
