// Tiles of rows, none of two experts: how a launch that cannot know the experts' rows finds its own.
#pragma once
#include "sparq_mx_experts.h"

namespace sparq {
namespace mx {

// A table in memory, made by a launch before (sparq_mx_experts.hip): its first unit holds the number of tiles, each further one a tile.
struct ExpertTile {
    int32_t row, rows, expert, unused;
};
// As many tiles as any division of the rows can make
inline int64_t most_tiles(int64_t rows, int experts, int tile) { return rows / tile + (rows < experts ? rows : experts); }
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
