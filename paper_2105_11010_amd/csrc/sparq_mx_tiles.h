// Tiles of rows, none of two experts: how a launch that cannot know the experts' rows finds its own.  Up to 64 experts each wavefront counts their tiles itself, a
// lane an expert, and keeps them in three registers; else, and where a kernel has no registers left, a launch before makes a table of the tiles (3 us).
#pragma once
#include "sparq_mx_experts.h"

namespace sparq {
namespace mx {

// A table in memory, made by a launch before (sparq_mx_experts.hip): its first unit holds the number of tiles, each further one a tile.
struct ExpertTile {
    int32_t row, rows, expert, unused;
};
// Tiles that n rows make (n + tile need not fit 32 bits)
inline constexpr int tiles_in(int n, int tile) { return n / tile + (n % tile != 0); }
// As many tiles as any division of the rows can make
inline int64_t most_tiles(int64_t rows, int experts, int tile) { return rows / tile + (rows < experts ? rows : experts); }
constexpr int kExpertsOfLanes = 64;
inline size_t table_bytes(int64_t rows, int experts) { return (size_t)round_up((most_tiles(rows, experts, 64) + 1) * (int64_t)sizeof(ExpertTile), 256); }
sparq_status launch_tiles(const int32_t* offsets, int experts, int64_t rows, int tile, void* table, hipStream_t stream);

#if defined(__HIPCC__)
// Expert e's rows, cut off at the borders
__device__ __forceinline__ void expert_rows(const int32_t* offsets, int e, int64_t rows, int& first, int& count) {
    const int most = (int)rows, a = offsets[e], b = offsets[e + 1];
    first = a < 0 ? 0 : a > most ? most : a;
    const int end = b > most ? most : b;
    count = end > first ? end - first : 0;
}
// A lane's expert: its rows, and the tiles of all experts up to it.  whole n > 0: of its first whole n rows alone; n < 0: of what is left behind whole -n rows.
struct LaneTiles {
    int first, rows, sum;
};
__device__ __forceinline__ LaneTiles tiles_of_lanes(const int32_t* offsets, int experts, int64_t rows, int tile, int whole = 0) {
    const int lane = threadIdx.x & 63;
    LaneTiles t = {0, 0, 0};
    if (lane < experts) expert_rows(offsets, lane, rows, t.first, t.rows);
    if (whole > 0) t.rows = t.rows / whole * whole;
    if (whole < 0) {
        const int n = t.rows / -whole * -whole;
        t.first += n;
        t.rows -= n;
    }
    t.sum = tiles_in(t.rows, tile);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int v = __shfl_up(t.sum, d);
        if (lane >= d) t.sum += v;
    }
    return t;
}
__device__ __forceinline__ int tile_count(const LaneTiles& t) { return __builtin_amdgcn_readlane(t.sum, 63); }
__device__ __forceinline__ ExpertTile expert_tile(const LaneTiles& t, int tile, uint32_t i) {
    const int e = __builtin_ctzll(__ballot((uint32_t)t.sum > i) | 1ull << 63), rows = __builtin_amdgcn_readlane(t.rows, e);
    const int in = ((int)i - (__builtin_amdgcn_readlane(t.sum, e) - tiles_in(rows, tile))) * tile;
    return {__builtin_amdgcn_readlane(t.first, e) + in, rows - in < tile ? rows - in : tile, e, 0};
}
// The table, by one workgroup, a thread an expert; sums: one of each wavefront.  Offsets that fall can make more tiles than fit 32 bits: `most` of them are written.
constexpr int kTableThreads = SPARQ_MX_EXPERTS_MOST;
__device__ __forceinline__ void write_tiles(const int32_t* offsets, int experts, int64_t rows, int tile, int most, ExpertTile* table, int64_t* sums) {
    const int e = threadIdx.x, lane = e & 63, wave = e >> 6;
    int first = 0, n = 0;
    if (e < experts) expert_rows(offsets, e, rows, first, n);
    const int tiles = tiles_in(n, tile);
    int64_t sum = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t v = __shfl_up(sum, d);
        if (lane >= d) sum += v;
    }
    if (lane == 63) sums[wave] = sum;
    __syncthreads();
    int64_t before = sum - tiles;
    for (int w = 0; w < wave; ++w) before += sums[w];
    const int64_t left = most - before;
    for (int i = 0; i < tiles && i < left; ++i) table[1 + before + i] = {first + i * tile, n - i * tile < tile ? n - i * tile : tile, e, 0};
    if (e == kTableThreads - 1) table[0] = {tiles < left ? (int)(before + tiles) : most, 0, 0, 0};
}
#if defined(__HIP_DEVICE_COMPILE__)
// (By the scalar cache: the table does not change while a kernel reads it.)
typedef __attribute__((address_space(4))) const int ConstantInt;
__device__ __forceinline__ int tile_count(const ExpertTile* table) { return *(ConstantInt*)table; }
__device__ __forceinline__ ExpertTile expert_tile(const ExpertTile* table, uint32_t i) {
    ConstantInt* const t = (ConstantInt*)(table + 1 + i);
    return {t[0], t[1], t[2], 0};
}
#endif
#endif

}  // namespace mx
}  // namespace sparq
