// The product of 4-bit operands for few rows: a decoding step, a serving batch.  y[m][n] = sum_k W[n][k] A[m][k] on
// v_mfma_scale_f32_16x16x128_f8f6f4, the weights the first operand: a lane feeds 32 values of one row, its block, and ends with four
// neighbouring n of one m.  Bound by the weights' way from memory.
// A workgroup makes 16 columns of y; its wavefronts divide the reduction in groups of 512 values (a row's 16 bytes of scales), and their sums
// are joined in LDS in the wavefronts' order.
// X not void: A is quantised on the way, by each wavefront for the groups it multiplies, and the next group's weights are asked for behind
// that; a further group waits for them and then for its part of A.
// A in codes: the loads are written a group ahead, but the compiler moves them behind the group before, and those of three times 16 rows
// among the matrix instructions, ten trips to memory a group.  What the loads' order could still give is in that.
// A call for 1 x 4096 x 4096 takes 3.9 us, of which a launch's 3 us and the wait for one round trip to memory are the most: 8.9 MB would pass in
// 1.3.  1 x 8192 x 8192 (36 MB of weights) takes 9.4, 3.8 TB/s, with A in codes 7.8; codes for 32 x 4096 x 4096 5.5.
#pragma once
#include <type_traits>

#include "sparq_mx_common.h"

namespace sparq {
namespace mx {

struct FewParams {
    const void* x;                       // [M][K] (quantised on the way), or
    const uint8_t *a, *as;               // codes and scales
    const uint8_t *w, *ws;
    const float* bias;
    int64_t ldx, ldy, code_pitch, scale_pitch;
    int32_t M, N, K, groups, last_step;  // groups of 512 values; the last step of 128
};

constexpr int kFewRows = 16;             // of W and of A an instruction takes
constexpr int kGroupRow = 256 + 16;      // bytes of a group of a row in LDS, and what keeps rows out of each other's banks
constexpr int kFewQuantised = kGroupRow + 16;       // with its scales

template <class O, class X, int MT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void few_rows_kernel(O* __restrict__ y, const FewParams p) {
    constexpr bool kQuantise = !std::is_void_v<X>;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * kFewRows, nw = n0 + r < p.N ? n0 + r : p.N - 1;
    const uint8_t *w = p.w + nw * p.code_pitch + 16 * g, *ws = p.ws + nw * p.scale_pitch;

    struct Group {
        v4i w[4], a[kQuantise ? 1 : MT][4];
        v4u ws, as[kQuantise ? 1 : MT];
    };
    auto fetch = [&](Group& o, int group) __attribute__((always_inline)) {
        group = group < p.groups ? group : p.groups - 1;     // (past the end: the last one again, for nobody)
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int step = 4 * group + s < p.last_step ? 4 * group + s : p.last_step;        // (a row's scales are zeros past its end)
            o.w[s] = *reinterpret_cast<const v4i*>(w + (int64_t)step * 64);
            if constexpr (!kQuantise) {
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const int m = 16 * i + r < p.M ? 16 * i + r : p.M - 1;
                    o.a[i][s] = *reinterpret_cast<const v4i*>(p.a + m * p.code_pitch + 16 * g + (int64_t)step * 64);
                }
            }
        }
        o.ws = *reinterpret_cast<const v4u*>(ws + (int64_t)group * 16);
        if constexpr (!kQuantise) {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int m = 16 * i + r < p.M ? 16 * i + r : p.M - 1;
                o.as[i] = *reinterpret_cast<const v4u*>(p.as + m * p.scale_pitch + (int64_t)group * 16);
            }
        }
    };
    v4f acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = v4f{};
    uint8_t* const mine = lds + wave * p.M * kFewQuantised;  // the wavefront's quantised rows
    const int ma = r < p.M ? r : 0;                          // (rows past the last one make results that are not stored)

    Group held;
    fetch(held, wave);
    for (int group = wave; group < p.groups; group += WAVES) {
        const Group now = held;
        if constexpr (kQuantise) {
            // (Four rows' loads at once, none in a branch that would have one wait for another: lanes past a row's whole runs read its first.)
            const int col = group * kScaleUnit + 8 * lane, n = p.K - col;
            const X* const x = static_cast<const X*>(p.x);
            for (int m0 = 0; m0 < p.M; m0 += 4) {
                float v[4][8];
                const X* row[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) row[i] = x + (m0 + i < p.M ? m0 + i : p.M - 1) * p.ldx;
                if (p.K >= 8) {
                    Raw8<X> raw[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        raw[i] = Raw8<X>{};
                        if (m0 + i < p.M) load_raw<false>(row[i] + (n >= 8 ? col : 0), raw[i]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (m0 + i >= p.M) break;
                        values_of(raw[i], v[i]);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[i][e] = n >= 8 ? v[i][e] : 0.0f;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
                }
                if (p.K % 8 && n > 0 && n < 8) {             // the lane that holds a row's end
                    X end[4][8];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < 8; ++e) end[i][e] = row[i][col + (e < n ? e : 0)];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[i][e] = e < n ? (float)end[i][e] : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (m0 + i >= p.M) break;
                    const uint32_t byte = scale4_of(block_top(v[i]));
                    uint8_t* to = mine + (m0 + i) * kFewQuantised;
                    *reinterpret_cast<uint32_t*>(to + 4 * lane) = codes4_of(v[i], byte);
                    if ((lane & 3) == 0) to[kGroupRow + (lane >> 2)] = (uint8_t)byte;
                }
            }
            wavefront_lds_fence();
        }
        fetch(held, group + WAVES);
        v4u as[MT];
        if constexpr (kQuantise) as[0] = *reinterpret_cast<const v4u*>(mine + ma * kFewQuantised + kGroupRow);
        else {
#pragma unroll
            for (int i = 0; i < MT; ++i) as[i] = now.as[i];
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const v8i wv = __builtin_shufflevector(now.w[s], now.w[s], 0, 1, 2, 3, -1, -1, -1, -1);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                v4i a;
                if constexpr (kQuantise) a = *reinterpret_cast<const v4i*>(mine + ma * kFewQuantised + s * 64 + 16 * g);
                else a = now.a[i][s];
                const v8i av = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
                acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, av, acc[i], 4, 4, 0, now.ws[s] >> (8 * g), 0, as[i][s] >> (8 * g));
            }
        }
        if constexpr (kQuantise) wavefront_lds_fence();
    }
    // ---- the wavefronts' sums
    __syncthreads();
    v4f* const sums = reinterpret_cast<v4f*>(lds);
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[(wave * MT + i) * 64 + lane] = acc[i];
    __syncthreads();
    for (int t = threadIdx.x; t < MT * 256; t += WAVES * 64) {
        const int i = t >> 8, from = (t >> 2) & 63, e = t & 3, m = 16 * i + (from & 15), n = n0 + 4 * (from >> 4) + e;
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) s += reinterpret_cast<const float*>(sums)[((k * MT + i) * 64 + from) * 4 + e];
        if (m < p.M && n < p.N) y[m * p.ldy + n] = (O)(s + (p.bias ? p.bias[n] : 0.0f));
    }
}

template <int WAVES, int MT>
inline size_t few_lds_bytes(int M, bool quantise) {
    const size_t sums = (size_t)WAVES * MT * 64 * 16, rows = quantise ? (size_t)WAVES * M * kFewQuantised : 0;
    return sums > rows ? sums : rows;
}

}  // namespace mx
}  // namespace sparq
