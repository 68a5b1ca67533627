// How a wavefront's results leave the matrix instruction's registers.
#pragma once
#include "sparq_mx_common.h"

namespace sparq {
namespace mx {

#if defined(__HIP_DEVICE_COMPILE__)
// acc[i][j]: 32 x 32 results each, the lane's row 32 j + lane % 32, its columns 32 i + 8 q + 4 (lane / 32) + e (element 4 q + e).
// They are rounded, turned in 32 x ROW_BYTES of LDS of the wavefront's own and stored in pieces of rows, 16 bytes a lane: stored from where
// they are, 8 bytes of 32 rows at a time, an 8192 x 8192 bf16 result took 100 us where whole rows take 30.  A row's 16-byte units are
// permuted by the row, or all rows would be written to the same banks.
// row0, col0: of the wavefront's first result; bias: one value a column, or a buffer without records for none.
template <class O, int FI, int FJ, int ROW_BYTES>
__device__ __forceinline__ void store_results(const v16f (&acc)[FI][FJ], O* out, int64_t ldo, int64_t row0, int64_t rows, int col0, int cols,
                                              const __amdgpu_buffer_rsrc_t bias, uint8_t* turn) {
    constexpr int PIECE = ROW_BYTES / (int)sizeof(O), PER = 16 / sizeof(O), UNITS = ROW_BYTES / 16, STEP = 64 / UNITS;
    static_assert(PIECE % 8 == 0 && FI * 32 % PIECE == 0, "pieces of whole runs of eight columns");
    const int lane = threadIdx.x & 63, c = lane & 31, g = lane >> 5;
    const int at = lane / UNITS, unit = lane % UNITS;
#pragma unroll
    for (int piece = 0; piece < FI * 32 / PIECE; ++piece) {
        v4f b[PIECE / 8];
#pragma unroll
        for (int run = 0; run < PIECE / 8; ++run)
            b[run] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(bias, (col0 + piece * PIECE + 8 * run + 4 * g) * 4, 0, 0));
        const int n = cols - col0 - piece * PIECE - unit * PER;
        O* const to_piece = out + (row0 + at) * ldo + col0 + piece * PIECE + unit * PER;
#pragma unroll
        for (int j = 0; j < FJ; ++j) {
#pragma unroll
            for (int run = 0; run < PIECE / 8; ++run) {
                const int i = (piece * PIECE + 8 * run) / 32, q = (piece * PIECE + 8 * run) % 32 / 8;
                O v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (O)(acc[i][j][4 * q + e] + b[run][e]);
                const int byte = (8 * run + 4 * g) * (int)sizeof(O);
                __builtin_memcpy(__builtin_assume_aligned(turn + c * ROW_BYTES + (((byte >> 4) ^ (c & (UNITS - 1))) << 4) + (byte & 15), sizeof(v)), v, sizeof(v));
            }
            wavefront_lds_fence();
#pragma unroll
            for (int r = 0; r < 32; r += STEP) {
                const v4u w = *reinterpret_cast<const v4u*>(turn + (r + at) * ROW_BYTES + ((unit ^ ((r + at) & (UNITS - 1))) << 4));
                if (row0 + 32 * j + r + at < rows && n > 0) {
                    O* to = to_piece + (int64_t)(32 * j + r) * ldo;
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
}
#endif

}  // namespace mx
}  // namespace sparq
