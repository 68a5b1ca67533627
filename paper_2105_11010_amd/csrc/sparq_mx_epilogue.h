// What becomes of a product's sums before they are rounded: bias, activation, residual, and their 8-bit form for the backward pass.
#pragma once
#include "sparq_mx_function.h"
#include "sparq_mx_store.h"

namespace sparq {
namespace mx {

struct Epilogue {
    const void* residual;                // of the results' type
    uint8_t *kept_codes, *kept_scales;   // NULL: not wanted
    int64_t ldr, code_pitch, scale_pitch;
    int32_t function, N128;

#if defined(__HIPCC__)
    // f(z) of eight values; one function a launch, so that the branch is the same for all
    template <class O>
    __device__ __forceinline__ void apply(float (&z)[8]) const {
        if (function == SPARQ_MX_SILU) {
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = mx::function<SPARQ_MX_SILU, sizeof(O) == 4>(z[e]);
        } else if (function == SPARQ_MX_GELU) {
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = mx::function<SPARQ_MX_GELU, sizeof(O) == 4>(z[e]);
        }
    }
    template <class O>
    __device__ __forceinline__ float apply(float z) const {
        if (function == SPARQ_MX_SILU) return mx::function<SPARQ_MX_SILU, sizeof(O) == 4>(z);
        return function == SPARQ_MX_GELU ? mx::function<SPARQ_MX_GELU, sizeof(O) == 4>(z) : z;
    }
    // Eight sums of a row, columns col and on, n of them there, four neighbouring lanes a block of 32.  inside: whether the row is.
    template <class O>
    __device__ __forceinline__ void finish(float (&z)[8], O* out, int64_t ldo, int64_t row, int col, int n, bool inside) const {
        if (kept_codes) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < n ? z[e] : 0.0f;
            const uint32_t byte = scale8_of(block_top(v));
            const v2u w = codes8_of(v, byte);
            if (inside && col < N128) *reinterpret_cast<v2u*>(kept_codes + row * code_pitch + col) = w;
            if (inside && (col & 31) == 0 && (col >> 5) < scale_pitch) kept_scales[row * scale_pitch + (col >> 5)] = (uint8_t)byte;
        }
        if (!inside || n <= 0) return;
        apply<O>(z);
        if (residual) {
            float r[8];
            load_upto8(static_cast<const O*>(residual) + row * ldr + col, n, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] += r[e];
        }
        store_upto8(out + row * ldo + col, n, z);
    }
#endif
#if defined(__HIP_DEVICE_COMPILE__)

    // A wavefront's sums, laid out as store_results (sparq_mx_store.h) has them.  They are turned as they are, in fp32, 32 columns of a row in 128 bytes of
    // LDS and ROWS rows at a time: a block of 32 is four neighbouring lanes then, and results leave as 64 (fp32: 128) bytes of a row.
    // tile_end: columns of the tile's end; past N the kept form's rows are filled up with zeros.
    template <class O, int FI, int FJ, int ROWS>
    __device__ __forceinline__ void store(const v16f (&acc)[FI][FJ], O* out, int64_t ldo, int64_t row0, int64_t rows, int col0, int cols, int tile_end,
                                          const __amdgpu_buffer_rsrc_t bias, uint8_t* turn) const {
        static_assert(ROWS == 32 || ROWS == 16);
        const int lane = threadIdx.x & 63, c = lane & 31, g = lane >> 5, at = lane >> 2, unit = 2 * (lane & 3);
#pragma unroll
        for (int i = 0; i < FI; ++i) {
            v4f b[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                b[q] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(bias, (col0 + 32 * i + 8 * q + 4 * g) * 4, 0, 0));
            const int col = col0 + 32 * i + 4 * unit, n = cols - col;
#pragma unroll
            for (int j = 0; j < FJ; ++j) {
#pragma unroll
                for (int part = 0; part < 32 / ROWS; ++part) {
                    if (ROWS == 32 || c / 16 == part) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            v4f z;
#pragma unroll
                            for (int e = 0; e < 4; ++e) z[e] = acc[i][j][4 * q + e] + b[q][e];
                            *reinterpret_cast<v4f*>(turn + c % ROWS * 128 + (((2 * q + g) ^ (c & 7)) << 4)) = z;
                        }
                    }
                    wavefront_lds_fence();
#pragma unroll
                    for (int r = 0; r < ROWS; r += 16) {
                        const uint8_t* from = turn + (r + at) * 128;
                        const v4f lo = *reinterpret_cast<const v4f*>(from + ((unit ^ (at & 7)) << 4)), hi = *reinterpret_cast<const v4f*>(from + (((unit + 1) ^ (at & 7)) << 4));
                        float z[8];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            z[e] = lo[e];
                            z[4 + e] = hi[e];
                        }
                        const int64_t row = row0 + 32 * j + ROWS * part + r + at;
                        finish<O>(z, out, ldo, row, col, n, row < rows);
                    }
                    wavefront_lds_fence();
                }
            }
        }
        // (tiles of 64 end before the codes' unit of 128 does, tiles of 256 before the scales' of 512)
        if (kept_codes && tile_end >= cols && col0 + FI * 32 == tile_end) {
            for (int r = lane; r < FJ * 32; r += 64) {
                const int64_t row = row0 + r;
                if (row >= rows) break;
                for (int k = tile_end; k < N128; k += 16) *reinterpret_cast<v4u*>(kept_codes + row * code_pitch + k) = v4u{};
                for (int64_t k = tile_end >> 5; k < scale_pitch; ++k) kept_scales[row * scale_pitch + k] = 0;
            }
        }
    }
#endif
};

}  // namespace mx
}  // namespace sparq
