// How a wavefront's results leave the matrix instruction's registers.
#pragma once
#include "sparq_mx_common.h"

namespace sparq {
namespace mx {

// LDS a wavefront turns 32 rows of COLS results in; rows 16 bytes apart beyond their length, which keeps rows out of each other's banks.
template <class O, int COLS> constexpr int kTurnPitch = COLS * (int)sizeof(O) + 16;
template <class O, int COLS> constexpr int kTurnBytes = 32 * kTurnPitch<O, COLS>;

#if defined(__HIP_DEVICE_COMPILE__)
// acc[i][j]: 32 x 32 results each, the lane's row 32 j + lane % 32, its columns 32 i + 8 q + 4 (lane / 32) + e (element 4 q + e).
// They are rounded, turned in the wavefront's own piece of LDS, 32 rows at a time, and stored in whole rows, 16 bytes a lane: stored from
// where they are, 8 bytes of 32 rows at a time, an 8192 x 8192 bf16 result took 100 us where this takes 30.
// row0, col0: of the wavefront's first result; bias: one value a column, or a buffer without records for none.
template <class O, int FI, int FJ>
__device__ __forceinline__ void store_results(const v16f (&acc)[FI][FJ], O* out, int64_t ldo, int64_t row0, int64_t rows, int col0, int cols,
                                              const __amdgpu_buffer_rsrc_t bias, uint8_t* turn) {
    constexpr int COLS = FI * 32, PITCH = kTurnPitch<O, COLS>, PER = 16 / sizeof(O), LANES = COLS / PER, STEP = 64 / LANES;
    const int lane = threadIdx.x & 63, c = lane & 31, g = lane >> 5;
    v4f b[FI][4];
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            b[i][q] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(bias, (col0 + 32 * i + 8 * q + 4 * g) * 4, 0, 0));
    const int at = lane / LANES, col = lane % LANES * PER, n = cols - col0 - col;
#pragma unroll
    for (int j = 0; j < FJ; ++j) {
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                O v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (O)(acc[i][j][4 * q + e] + b[i][q][e]);
                __builtin_memcpy(__builtin_assume_aligned(turn + c * PITCH + (32 * i + 8 * q + 4 * g) * sizeof(O), 4 * sizeof(O)), v, sizeof(v));
            }
        wavefront_lds_fence();
#pragma unroll
        for (int r = 0; r < 32; r += STEP) {
            const v4u w = *reinterpret_cast<const v4u*>(turn + (r + at) * PITCH + col * sizeof(O));
            const int64_t row = row0 + 32 * j + r + at;
            if (row < rows && n > 0) {
                O* to = out + row * ldo + col0 + col;
                if (n >= PER) __builtin_memcpy(to, &w, 16);
                else {
                    O v[PER];
                    __builtin_memcpy(v, &w, 16);
#pragma unroll
                    for (int e = 0; e < PER; ++e)
                        if (e < n) to[e] = v[e];
                }
            }
        }
        wavefront_lds_fence();
    }
}
#endif

}  // namespace mx
}  // namespace sparq
