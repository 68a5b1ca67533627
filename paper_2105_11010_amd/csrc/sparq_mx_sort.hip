// The router's choices sorted by expert (include/sparq_mx_experts.h).
#include "sparq_mx_experts.h"

namespace sparq {
namespace mx {

// A counting sort that keeps the order of equal keys.  A wavefront has a range of slots, kAhead times 64 of them in registers at a time: it counts them by expert
// in LDS, and once the counts of all ranges before its own are known, for each expert, it takes 64 slots at a time; a slot's rank among the lanes with the
// same expert is the number of such lanes below, found by one ballot a bit of the expert's number.  Slots refused are those of one expert more, the last.
// Bound by waiting: for the slots, the other workgroups' counts, and as many rounds of ballots as a range has 64s.  262144 slots among 256 experts 13.2 us (4 and 11 in
// its two kernels; 3 MB, 0.5 at memory's pace), 16384 among 8 8.6.
struct SortParams {
    const int32_t* expert;
    int32_t *offsets, *place, *order;
    int32_t* counts;             // [workgroups][experts + 1], of more workgroups than one
    int32_t slots, experts, range;               // slots of a wavefront (whole kAhead 64s)
};
constexpr int kAhead = 2;                    // (us, one -> two -> four: 16384 slots among 8 experts 7.8, 8.6, 9.9; 262144 among 256 16.8, 13.2, 13.1)

// Lanes' buckets of kAhead times 64 slots from s on (-1: past the end)
__device__ __forceinline__ void buckets_of(const SortParams& p, int64_t s, int (&key)[kAhead]) {
    const int lane = threadIdx.x & 63;
    int e[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) e[i] = p.expert[s + 64 * i + lane < p.slots ? s + 64 * i + lane : p.slots - 1];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) key[i] = s + 64 * i + lane >= p.slots ? -1 : (unsigned)e[i] < (unsigned)p.experts ? e[i] : p.experts;
}
__device__ __forceinline__ void count_range(const SortParams& p, int64_t first, int32_t* counts, int (&key)[kAhead]) {
    for (int64_t s = first; s < first + p.range && s < p.slots; s += 64 * kAhead) {
        buckets_of(p, s, key);
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (key[i] >= 0) atomicAdd(&counts[key[i]], 1);
    }
}

// Counts of a workgroup's slots
template <int WAVES>
__global__ __launch_bounds__(WAVES * 64) void sort_count_kernel(const SortParams p) {
    extern __shared__ int32_t counts[];
    const int buckets = p.experts + 1;
    for (int i = threadIdx.x; i < buckets; i += WAVES * 64) counts[i] = 0;
    __syncthreads();
    int key[kAhead];
    count_range(p, (int64_t)(blockIdx.x * WAVES + (threadIdx.x >> 6)) * p.range, counts, key);
    __syncthreads();
    for (int i = threadIdx.x; i < buckets; i += WAVES * 64) p.counts[(int64_t)blockIdx.x * buckets + i] = counts[i];
}

template <int WAVES, bool MANY>
__global__ __launch_bounds__(WAVES * 64) void sort_kernel(const SortParams p) {
    constexpr int THREADS = WAVES * 64;
    // [WAVES][buckets] counts, then the wavefronts' next rows; [buckets] the counts before the workgroup's (MANY) and all of them; [WAVES] sums
    extern __shared__ int32_t lds[];
    const int buckets = p.experts + 1, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t *const mine = lds + wave * buckets, *const before = lds + WAVES * buckets, *const all = before + buckets, *const sums = all + buckets;
    for (int i = threadIdx.x; i < (WAVES + 2) * buckets; i += THREADS) lds[i] = 0;
    __syncthreads();
    const int64_t first = (int64_t)(blockIdx.x * WAVES + wave) * p.range;
    int key[kAhead];                             // of a range no longer than these, for good
    count_range(p, first, mine, key);
    __syncthreads();
    // Counts before each wavefront, and all of them: of other workgroups by as many threads a bucket as there are, 16 workgroups' on their way at a time
    if constexpr (MANY) {
        const int parts = THREADS / buckets > 1 ? THREADS / buckets : 1;
        for (int i = threadIdx.x; i < parts * buckets; i += THREADS) {
            const int part = i / buckets, e = i - part * buckets;
            int n_before = 0, total = 0;
            for (int b0 = part; b0 < (int)gridDim.x; b0 += 16 * parts) {
                int n[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) n[j] = p.counts[(int64_t)(b0 + j * parts < (int)gridDim.x ? b0 + j * parts : 0) * buckets + e];
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int b = b0 + j * parts;
                    if (b < (int)gridDim.x) total += n[j];
                    if (b < (int)blockIdx.x) n_before += n[j];
                }
            }
            atomicAdd(&before[e], n_before);
            atomicAdd(&all[e], total);
        }
        __syncthreads();
    }
    for (int e = threadIdx.x; e < buckets; e += THREADS) {
        int sum = MANY ? before[e] : 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int n = lds[w * buckets + e];
            lds[w * buckets + e] = sum;
            sum += n;
        }
        if (!MANY) all[e] = sum;
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
    for (int64_t s0 = first; s0 < first + p.range && s0 < p.slots; s0 += 64 * kAhead) {
        if (p.range > 64 * kAhead) buckets_of(p, s0, key);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (s0 + 64 * i >= p.slots) break;
            const int64_t s = s0 + 64 * i + lane;
            const bool there = key[i] >= 0;
            uint64_t same = __ballot(there);
            for (int b = 0; b < bits; ++b) {
                const uint64_t set = __ballot(key[i] >> b & 1);
                same &= key[i] >> b & 1 ? set : ~set;
            }
            const int rank = __popcll(same & ((1ull << lane) - 1));
            if (there) {
                const int row = mine[key[i]] + rank;
                p.place[s] = key[i] < p.experts ? row : -1;
                if (p.order) p.order[row] = key[i] < p.experts ? (int)s : -1;
            }
            wavefront_lds_fence();
            if (there && rank == 0) mine[key[i]] += __popcll(same);
            wavefront_lds_fence();
        }
    }
}

// One workgroup for a few thousand slots (4096 among 8 experts 6.5 us, 300 4.4; 8192 among 1024 in one 16.1, in two 11.8); more take two launches,
// the first of which counts: as few slots a workgroup as leave no more than 256 of them, whose counts each adds up.
struct SortPlan {
    int waves, range, blocks;
    size_t bytes;
};
static SortPlan sort_plan(int64_t slots, int experts) {
    SortPlan p = {};
    constexpr int least = 64 * kAhead;
    const int most = experts <= 512 ? 16 : 8;                // (LDS)
    p.waves = slots <= least ? 1 : most;
    const int64_t ranges = (slots + least - 1) / least, wanted = slots <= 4096 ? p.waves : most * 256;
    p.range = ranges > wanted ? (int)round_up((slots + wanted - 1) / wanted, least) : least;
    p.blocks = slots == 0 ? 1 : (int)((slots + (int64_t)p.range * p.waves - 1) / ((int64_t)p.range * p.waves));
    p.bytes = p.blocks > 1 ? (size_t)round_up((int64_t)p.blocks * (experts + 1) * 4, 256) : 0;
    return p;
}
static bool sort_sizes_ok(int64_t slots, int experts) { return slots >= 0 && experts >= 1; }
static bool sort_countable(int64_t slots, int experts) { return slots <= 1 << 30 && experts <= SPARQ_MX_EXPERTS_MOST; }

template <int WAVES>
static sparq_status launch_sort(const SortParams& p, int blocks, hipStream_t stream) {
    const int buckets = p.experts + 1, lds_bytes = ((WAVES + 2) * buckets + WAVES) * 4;
    if (blocks == 1) {
        sort_kernel<WAVES, false><<<1, WAVES * 64, lds_bytes, stream>>>(p);
        return launch_status();
    }
    sort_count_kernel<WAVES><<<blocks, WAVES * 64, buckets * 4, stream>>>(p);
    const sparq_status counted = launch_status();
    if (counted != SPARQ_OK) return counted;
    sort_kernel<WAVES, true><<<blocks, WAVES * 64, lds_bytes, stream>>>(p);
    return launch_status();
}

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
    const SortParams p = {expert, offsets, place, order, static_cast<int32_t*>(workspace), (int32_t)slots, experts, plan.range};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return plan.waves == 1 ? launch_sort<1>(p, plan.blocks, s) : plan.waves == 8 ? launch_sort<8>(p, plan.blocks, s) : launch_sort<16>(p, plan.blocks, s);
}
