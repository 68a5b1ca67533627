// What becomes of a product's sums before they are rounded: bias, activation, residual, and their 8-bit form for the backward pass.
#pragma once
#include "../../include/sparq_mx_experts.h"
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

    // A wavefront's sums, laid out as store_results (sparq_mx_store.h) has them: a lane has, of 32 x 32, four columns of every eight of one row, and the lane 32
    // further the other four.  Eight exchanges between the two leave either with sixteen neighbouring columns, in fp32, of which everything is made
    // in registers; results leave as 32 (fp32: 64) bytes a lane, the four pieces of a row one after the other, the residual's next piece on its way.
    // (Turned in LDS, 32 columns at a time, a tile's end had three times as many waits: 16384 x 4096 x 2048 150 us, of which the product's own is 100.)
    // tile_end: columns of the tile's end; past N the kept form's rows are filled up with zeros.  shared: 4 FI 32 bytes of LDS of the wavefront's own.
    template <int F, class O, int FI, int FJ>
    __device__ __forceinline__ void store(const v16f (&acc)[FI][FJ], O* out, int64_t ldo, int64_t row0, int64_t rows, int col0, int cols, int tile_end,
                                          const float* bias, uint8_t* shared) const {
        const int lane = threadIdx.x & 63, c = lane & 31, g = lane >> 5;
        if (row0 >= rows || (col0 >= cols && !kept_codes)) return;
        float* const its_bias = reinterpret_cast<float*>(shared);
        if (bias) {                                          // (asked for here, and not piece by piece behind the stores, each of which it would wait for)
#pragma unroll
            for (int k = lane; k < FI * 32; k += 64) its_bias[k] = bias[col0 + k < cols ? col0 + k : cols - 1];
            wavefront_lds_fence();
        }
        const bool whole = col0 + FI * 32 <= cols;
        const int64_t last = rows - 1;
        constexpr int kWords = 4 * (int)sizeof(O);           // of sixteen columns
        struct Piece {
            uint32_t w[kWords];
        };
        // sixteen columns of row 32 j + c: piece i of the row
        auto fetch = [&](int i, int j, Piece& r) __attribute__((always_inline)) {
            const int64_t row = row0 + 32 * j + c;
            const O* from = static_cast<const O*>(residual) + (row < last ? row : last) * ldr + col0 + 32 * i + 16 * g;
#pragma unroll
            for (int h = 0; h < kWords / 4; ++h) {
                const v4u w = word_at<false>(from + h * (16 / (int)sizeof(O)));
#pragma unroll
                for (int e = 0; e < 4; ++e) r.w[4 * h + e] = w[e];
            }
        };
        Piece next;
        if (residual && whole) fetch(0, 0, next);
#pragma unroll
        for (int j = 0; j < FJ; ++j) {
            const int64_t row = row0 + 32 * j + c;
            const bool inside = row < rows;
            uint32_t bytes = 0;                              // of the kept form's scales
#pragma unroll
            for (int i = 0; i < FI; ++i) {
                const Piece now = next;
                if (residual && whole && j * FI + i + 1 < FI * FJ) fetch((i + 1) % FI, j + (i + 1) / FI, next);
                float z[16];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const auto pair = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i][j][4 * h + e]), __float_as_uint(acc[i][j][8 + 4 * h + e]), false, false);
                        z[8 * h + e] = __uint_as_float(pair[0]);
                        z[8 * h + 4 + e] = __uint_as_float(pair[1]);
                    }
                if (bias) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const v4f b = *reinterpret_cast<const v4f*>(its_bias + 32 * i + 16 * g + 4 * q);
#pragma unroll
                        for (int e = 0; e < 4; ++e) z[4 * q + e] += b[e];
                    }
                }
                const int col = col0 + 32 * i + 16 * g, n = cols - col;
                if (kept_codes) {
                    if (!whole) {                            // (columns past N, which are zeros in the kept form and are not stored)
#pragma unroll
                        for (int e = 0; e < 16; ++e) z[e] = e < n ? z[e] : 0.0f;
                    }
                    uint32_t top = 0;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const uint32_t m = __float_as_uint(z[e]) & 0x7FFFFFFFu;
                        top = m > top ? m : top;
                    }
                    const auto other = __builtin_amdgcn_permlane32_swap(top, top, false, false);
                    const uint32_t a = other[0], b = other[1], byte = scale8_of(a > b ? a : b);
                    v4u w;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float v[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = z[8 * h + e];
                        const v2u half = codes8_of(v, byte);
                        w[2 * h] = half[0];
                        w[2 * h + 1] = half[1];
                    }
                    bytes |= byte << (8 * i);
                    if (inside && col < N128) *reinterpret_cast<v4u*>(kept_codes + row * code_pitch + col) = w;
                }
                if constexpr (F != SPARQ_MX_NONE) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) z[e] = mx::function<F, sizeof(O) == 4>(z[e]);
                }
                O* const to = out + row * ldo + col;
                if (residual) {
                    if (whole) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            if constexpr (sizeof(O) == 4) z[e] += __uint_as_float(now.w[e]);
                            else {
                                const uint16_t h = (uint16_t)(now.w[e >> 1] >> (16 * (e & 1)));
                                z[e] += (float)__builtin_bit_cast(O, h);
                            }
                        }
                    } else if (inside) {
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (e < n) z[e] += (float)static_cast<const O*>(residual)[row * ldr + col + e];
                    }
                }
                if (inside && (whole || n >= 16)) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float v[8] = {z[8 * h], z[8 * h + 1], z[8 * h + 2], z[8 * h + 3], z[8 * h + 4], z[8 * h + 5], z[8 * h + 6], z[8 * h + 7]};
                        store8(to + 8 * h, v);
                    }
                } else if (inside) {
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (e < n) to[e] = (O)z[e];
                }
            }
            // (a row's scales of this tile, or those of them that are inside the row: rows are whole units of sixteen)
            if (kept_codes && inside && g == 0) {
                uint8_t* const to = kept_scales + row * scale_pitch + (col0 >> 5);
#pragma unroll
                for (int i = 0; i < FI; ++i)
                    if ((col0 >> 5) + i < scale_pitch) to[i] = (uint8_t)(bytes >> (8 * i));
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
