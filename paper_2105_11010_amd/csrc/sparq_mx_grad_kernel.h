// The product's gradients: out[j][k] = sum_r dy(j, r) V[r][k] on v_mfma_f32_32x32x16_bf16.
//   dx: j = m, r = n, V = the 4-bit weights;   dw: j = n, r = m, V = the 8-bit checkpoint.
// V's codes and scales go through registers into bf16 (their values are bf16 exactly: at most eight significand bits and a
// power of two) and, turned so that the reduction index is the fast one, into LDS; dy goes the same way, as one bf16 part
// (bf16), two (fp16) or three (fp32) whose sum is the value.
// A workgroup of four wavefronts makes TJ x TK results in steps of 64 products, a wavefront a quarter of them.  What is here takes steps of
// any kind, one after the other, with checked loads: the last step of a reduction, and calls whose rows lie too far apart for
// sparq_mx_grad_wide_kernel.h, which takes the others.
#pragma once
#include <type_traits>

#include "sparq_mx_store.h"

namespace sparq {
namespace mx {

struct GradParams {
    const void* dy;
    const uint8_t *codes, *scales;
    int64_t lddy, code_pitch, scale_pitch, ldo;
    int64_t J, R;                        // results [J][K], sums of R products
    int64_t part_stride;                 // results of a part of the reduction lie this far apart (parts > 1)
    int32_t K, K128;                     // row length, the same in whole units of codes
    int32_t tiles_j, tiles_k;
    int32_t steps_per_part;              // steps of 64 products
    float* column_sums;                  // [slabs][J], of dy [R][J] (dw), by workgroups past the tiles', or by a launch before
    int64_t slab;                        // rows of one
    int32_t slabs;
    int64_t s_whole;                     // steps before this one are read without checks
};

constexpr int kGradThreads = 256;
constexpr int kGradStep = 64;

// The bf16 parts of a value: their sum is the value (8 significand bits a part; fp16 has 11, fp32 24).  Each is what is left cut off behind its
// eighth bit, not rounded: fp32's values above bf16's largest would be rounded to infinity.
template <class T> inline constexpr int kParts = sizeof(T) == 4 ? 3 : 2;
template <> inline constexpr int kParts<__bf16> = 1;
template <int P>
__device__ __forceinline__ void split(float v, float (&part)[P]) {
    part[0] = v;
#pragma unroll
    for (int i = 1; i < P; ++i) {
        const float whole = part[i - 1], cut = __uint_as_float(__float_as_uint(whole) & 0xFFFF0000u);
        part[i - 1] = cut;
        part[i] = __builtin_fabsf(whole) == __builtin_inff() ? 0.0f : whole - cut;       // infinity: nothing to add
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) { return pack2(a, b, __bf16{}); }

// C neighbouring elements
template <int BYTES> struct Word;
template <> struct Word<1> { typedef uint8_t Type; };
template <> struct Word<2> { typedef uint16_t Type; };
template <> struct Word<4> { typedef uint32_t Type; };
template <> struct Word<8> { typedef v2u Type; };

// 16-byte unit of a tile: rows of 64 bf16 are eight of them, permuted so that neither eight rows at one place of the reduction
// (the matrix operands' reads) nor every eighth row (the writes of turned blocks) meet in the same banks.
__device__ __forceinline__ int unit_at(int row, int chunk) { return row * 8 + (chunk ^ ((row ^ (row >> 3)) & 7)); }

// An element of type T in a register's low (half 0) or high half
template <class T>
__device__ __forceinline__ float element(uint32_t w, int half) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w);
    else {
        const uint16_t h = (uint16_t)(half ? w >> 16 : w);
        return (float)__builtin_bit_cast(T, h);
    }
}
// COUNT neighbouring elements as they lie in memory, of which the first n are there.  Without branches, which would have one load wait for
// another: what is not there is read from `safe` and left out.
template <class T, int COUNT>
__device__ __forceinline__ void fetch(uint32_t (&w)[COUNT * sizeof(T) / 4], const T* at, int64_t n, const T* safe) {
    typedef std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t> Bits;
    Bits v[COUNT];
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = *reinterpret_cast<const Bits*>(i < n ? at + i : safe);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = i < n ? v[i] : (Bits)0;
#pragma unroll
    for (int i = 0; i < COUNT * (int)sizeof(T) / 4; ++i) {
        if constexpr (sizeof(T) == 4) w[i] = v[i];
        else w[i] = v[2 * i] | (uint32_t)v[2 * i + 1] << 16;
    }
}

// dy's side of a tile.  TURN: dy [r][j], a thread takes 8 r x N j; else dy [j][r], a thread takes N runs of 8 r.
template <class T, int TJ, bool TURN>
struct DyTile {
    static constexpr int P = kParts<T>, N = TJ / 32;
    static constexpr int kRuns = TURN ? 8 : N, kLength = TURN ? N : 8, kPer = 4 / sizeof(T);        // elements a word
    uint32_t v[kRuns][kLength / kPer];

    __device__ __forceinline__ void load(const GradParams& p, int64_t j0, int64_t r0) {
        const T* dy = static_cast<const T*>(p.dy);
        const int t = threadIdx.x;
        if constexpr (TURN) {
            const int64_t j = j0 + (t & 31) * N, r = r0 + (t >> 5) * 8;
            const T* at = dy + r * p.lddy + j;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                fetch<T, N>(v[i], at, r + i < p.R ? p.J - j : 0, dy);
                at += p.lddy;
            }
        } else {
            const int64_t r = r0 + (t & 7) * 8;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                int64_t j = j0 + (t >> 3) + 32 * i;
                j = j < p.J ? j : p.J - 1;                   // (rows past the last one make results that are not stored)
                fetch<T, 8>(v[i], dy + j * p.lddy + r, p.R - r, dy);
            }
        }
    }
    // column or run c into the parts' tiles
    __device__ __forceinline__ void store(v4u* lds, int c) const {
        const int t = threadIdx.x;
        const int at_row = TURN ? (t & 31) * N + c : (t >> 3) + 32 * c, chunk = TURN ? t >> 5 : t & 7;
        const int at = unit_at(at_row, chunk);
        if constexpr (P == 1) {
            v4u w;
#pragma unroll
            for (int a = 0; a < 4; ++a)
                w[a] = TURN ? __builtin_amdgcn_perm(v[2 * a + 1][c / 2], v[2 * a][c / 2], c & 1 ? 0x07060302u : 0x05040100u) : v[c][a];
            lds[at] = w;
        } else {
            float part[8][P];
#pragma unroll
            for (int a = 0; a < 8; ++a) split<P>(TURN ? element<T>(v[a][c / kPer], c % kPer) : element<T>(v[c][a / kPer], a % kPer), part[a]);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                v4u w;
#pragma unroll
                for (int a = 0; a < 4; ++a) w[a] = pack_bf16(part[2 * a][i], part[2 * a + 1][i]);
                lds[i * TJ * 8 + at] = w;
            }
        }
    }
};

// The coded side: a thread takes 8 r x COLS k.
template <int BITS, int TK>
struct CodedTile {
    static constexpr int N = TK / 32;
    typedef typename Word<N * BITS / 8>::Type Raw;
    Raw raw[8];
    uint32_t scale[8];

    __device__ __forceinline__ void load(const GradParams& p, int k0, int64_t r0) {
        const int t = threadIdx.x;
        int k = k0 + (t & 31) * N;
        k = k < p.K128 ? k : p.K128 - N;                     // (columns past the last one make results that are not stored)
        const int64_t r = r0 + (t >> 5) * 8;
        const uint8_t *at = p.codes + r * p.code_pitch + k * BITS / 8, *sc = p.scales + r * p.scale_pitch + (k >> 5);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool there = r + i < p.R;
            raw[i] = *reinterpret_cast<const Raw*>(there ? at + i * p.code_pitch : p.codes);
            scale[i] = *(there ? sc + i * p.scale_pitch : p.scales);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool there = r + i < p.R;
            raw[i] = there ? raw[i] : Raw{};
            scale[i] = there ? scale[i] : 127u;
        }
    }
    // columns 2 q and 2 q + 1
    __device__ __forceinline__ void store(v4u* lds, int q) const {
        const int t = threadIdx.x, row = (t & 31) * N + 2 * q, chunk = t >> 5;
        v4u even, odd;
        if constexpr (BITS == 4) {
            uint32_t pair[8];                                // columns 2 q (low) and 2 q + 1 of a row
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                pair[i] = pair4_of(raw[i], scale_operand(scale[i]), q);
            }
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                even[a] = __builtin_amdgcn_perm(pair[2 * a + 1], pair[2 * a], 0x05040100u);
                odd[a] = __builtin_amdgcn_perm(pair[2 * a + 1], pair[2 * a], 0x07060302u);
            }
        } else {
            float v[8][2];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t w;
                if constexpr (N == 8) w = raw[i][q >> 1];
                else w = (uint32_t)raw[i];
                const float s = unit8_of(scale[i]);
                v[i][0] = (float)(int8_t)(w >> (16 * (q & 1))) * s;
                v[i][1] = (float)(int8_t)(w >> (16 * (q & 1) + 8)) * s;
            }
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                even[a] = pack_bf16(v[2 * a][0], v[2 * a + 1][0]);
                odd[a] = pack_bf16(v[2 * a][1], v[2 * a + 1][1]);
            }
        }
        lds[unit_at(row, chunk)] = even;
        lds[unit_at(row + 1, chunk)] = odd;
    }
};

// What a wavefront of four multiplies: a quarter of a tile, FK x FJ results of 32 x 32.
template <int P, int TJ, int TK>
struct Products {
    static constexpr int FJ = TJ / 64, FK = TK / 64;
    v16f acc[FK][FJ];
    int wj, wk;                                              // the wavefront's first row and column of the tile

    __device__ __forceinline__ Products() {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wj = (wave >> 1) * (TJ / 2);
        wk = (wave & 1) * (TK / 2);
#pragma unroll
        for (int a = 0; a < FK; ++a)
#pragma unroll
            for (int b = 0; b < FJ; ++b) acc[a][b] = v16f{};
    }
    // products of quarter q of a tile in LDS
    __device__ __forceinline__ void multiply(const v4u* tile, int q) {
        const int c = threadIdx.x & 31, g = (threadIdx.x >> 5) & 1;
        const v4u* tile_k = tile + P * TJ * 8;
        v8bf a[FK], b[P][FJ];
#pragma unroll
        for (int f = 0; f < FK; ++f) a[f] = __builtin_bit_cast(v8bf, tile_k[unit_at(wk + 32 * f + c, 2 * q + g)]);
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int f = 0; f < FJ; ++f) b[i][f] = __builtin_bit_cast(v8bf, tile[i * TJ * 8 + unit_at(wj + 32 * f + c, 2 * q + g)]);
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int x = 0; x < FK; ++x)
#pragma unroll
                for (int y = 0; y < FJ; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[x], b[i][y], acc[x][y], 0, 0, 0);
    }
};
// Sums of dy's columns, rows begin to end: a workgroup takes kColumns of them, eight a lane, and kRows rows at a time.
template <class T, int THREADS>
struct ColumnSums {
    static constexpr int kColumns = THREADS == 1024 ? 64 : 32, kLanes = kColumns / 8, kRows = THREADS / kLanes, kSlices = THREADS / kColumns;
    static constexpr int kAhead = THREADS == 1024 ? 4 : 2;                     // (beside a product's tiles: in the registers these have)
    static constexpr int kPitch = kColumns + 4, kFloats = kRows * kPitch;
    static __device__ __forceinline__ void run(const T* __restrict__ dy, int64_t ld, int64_t begin, int64_t end, int n, int first, float* __restrict__ sum, float* shared) {
        const int t = threadIdx.x, x = t % kLanes, r0 = t / kLanes, c = first + 8 * x;
        float s[8] = {};
        if (c < n)
            for (int64_t r = begin + r0; r < end; r += kAhead * kRows) {
                float v[kAhead][8];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) load_upto8(dy + (r + u * kRows) * ld + c, r + u * kRows < end ? n - c : 0, v[u]);
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[i] += v[u][i];
            }
#pragma unroll
        for (int i = 0; i < 8; ++i) shared[r0 * kPitch + 8 * x + i] = s[i];
        __syncthreads();
        // kSlices threads a column, eight rows each, then one
        const int col = t % kColumns, part = t / kColumns;
        float total = 0.0f;
#pragma unroll
        for (int i = 0; i < kRows / kSlices; ++i) total += shared[(part * (kRows / kSlices) + i) * kPitch + col];
        __syncthreads();
        shared[part * kPitch + col] = total;
        __syncthreads();
        if (part != 0 || first + col >= n) return;
#pragma unroll
        for (int i = 1; i < kSlices; ++i) total += shared[i * kPitch + col];
        sum[first + col] = total;
    }
};

// Steps that are not whole, or whose loads would not be: checked loads, one step after the other.
template <class T, bool DW, int TJ, int TK>
__device__ __forceinline__ void multiply_rest(Products<kParts<T>, TJ, TK>& products, const GradParams& p, v4u* lds, int64_t j0, int k0, int64_t s, int64_t s_end) {
    typedef DyTile<T, TJ, DW> Dy;
    typedef CodedTile<DW ? 8 : 4, TK> Coded;
    for (; s < s_end; ++s) {
        Dy dy;
        Coded coded;
        dy.load(p, j0, s * kGradStep);
        coded.load(p, k0, s * kGradStep);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TJ / 32; ++i) dy.store(lds, i);
#pragma unroll
        for (int i = 0; i < TK / 64; ++i) coded.store(lds + Dy::P * TJ * 8, i);
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 4; ++q) products.multiply(lds, q);
    }
}

}  // namespace mx
}  // namespace sparq
