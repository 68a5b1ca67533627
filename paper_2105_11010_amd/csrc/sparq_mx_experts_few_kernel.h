// The experts' product for few rows each: a decoding step, a serving batch.  y[m][n] = r[m][n] + f(sum_k W[e][n][k] A[m][k] + b[e][n]) on
// v_mfma_scale_f32_16x16x128_f8f6f4, the weights the first operand, as in sparq_mx_few_kernel.h.  Bound by the weights' way from memory.
// The experts' rows are divided into pieces of at most 16 MT; a workgroup finds the rows of its piece from the offsets (a lane an expert), and makes 16 columns of
// their results after the other, `blocks` times: its wavefronts divide the reduction in groups of 512 values (a row's 16 bytes of scales), and their sums are
// joined in LDS in the wavefronts' order.  The next two blocks' weights are on their way meanwhile, and where each wavefront has one group, its part of A stays
// in registers: read, or quantised, once for all blocks.
// 16 rows, 11 of 16 experts with weights of 2048 x 4096: 12.2 us (47 MB, 7.1 at memory's pace, and what any launch takes); when it was chosen, side by side, 13.9, with a
// block a workgroup 16.7, with one on its way and not two 14.1; two experts 5.0.
#pragma once
#include <type_traits>

#include "sparq_mx_epilogue.h"
#include "sparq_mx_tiles.h"

namespace sparq {
namespace mx {

struct ExpertFewParams {
    const void* x;                       // [M][K] (quantised on the way; no more groups than wavefronts), or
    const uint8_t *a, *as;               // codes and scales
    const uint8_t *w, *ws;
    const float* bias;
    const int32_t* offsets;              // NULL: one expert, all rows (M, at most 16 MT)
    int64_t ldx, ldy, code_pitch, scale_pitch, M;
    int32_t N, K, groups, last_step;     // groups of 512 values; the last step of 128
    int32_t experts, blocks;             // blocks: of 16 columns a workgroup makes
    Epilogue epilogue;
};

constexpr int kFewColumns = 16;          // rows of W, and of A, an instruction takes
constexpr int kFewRow = 256 + 16 + 16;   // bytes of a quantised group of a row in LDS: codes, what keeps rows out of each other's banks, scales

#if defined(__HIPCC__)
// The rows of piece `index` of the pieces of at most `most` rows that the experts' rows are divided into; false: there are fewer.  A lane an expert.
__device__ __forceinline__ bool find_piece(const int32_t* offsets, int experts, int64_t rows, int most, uint32_t index, int& row0, int& count, int& expert) {
    const int lane = threadIdx.x & 63;
    uint32_t before = 0;
    for (int e0 = 0; e0 < experts; e0 += 64) {
        int first = 0, n = 0;
        if (e0 + lane < experts) expert_rows(offsets, e0 + lane, rows, first, n);
        const uint32_t pieces = (uint32_t)(n + most - 1) / (uint32_t)most;
        uint32_t sum = pieces;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t v = __shfl_up(sum, d);
            if (lane >= d) sum += v;
        }
        const uint64_t past = __ballot(before + sum > index);
        if (past) {
            const int at = __builtin_ctzll(past);
            const int in = (int)(index - before - (uint32_t)__builtin_amdgcn_readlane((int)(sum - pieces), at)) * most;
            row0 = __builtin_amdgcn_readlane(first, at) + in;
            count = __builtin_amdgcn_readlane(n, at) - in;
            count = count < most ? count : most;
            expert = e0 + at;
            return true;
        }
        before += (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
    }
    return false;
}

// SINGLE: no more groups than wavefronts.
template <class O, class X, int MT, int WAVES, bool SINGLE>
__global__ __launch_bounds__(WAVES * 64) void experts_few_kernel(O* __restrict__ y, const ExpertFewParams p) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool kQuantise = !std::is_void_v<X>;
    static_assert(!kQuantise || (MT == 1 && SINGLE));
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    int M = (int)p.M, row0 = 0, expert = 0;
    if (p.offsets && !find_piece(p.offsets, p.experts, p.M, 16 * MT, blockIdx.y, row0, M, expert)) return;
    const int block0 = blockIdx.x * p.blocks, all = (p.N + kFewColumns - 1) / kFewColumns, blocks = all - block0 < p.blocks ? all - block0 : p.blocks;
    const uint8_t *const w = p.w + (int64_t)expert * p.N * p.code_pitch, *const ws = p.ws + (int64_t)expert * p.N * p.scale_pitch;

    struct Weights {
        v4i w[4];
        v4u ws;
    };
    struct Rows {
        v4i a[MT][4];
        v4u as[MT];
    };
    // Columns past N, blocks past the last one and groups past the row's lie past the buffer's end: they come as zeros, without a request.  (Of no rows the scalar
    // part of the offset is 0 too: what it would leave of a size of 0, taken as a number without a sign, is no end.)
    auto fetch = [&](Weights& o, int block, int group) __attribute__((always_inline)) {
        const int n0 = (block0 + block) * kFewColumns, rows = block >= blocks || group >= p.groups ? 0 : p.N - n0 < kFewColumns ? p.N - n0 : kFewColumns;
        const auto buffer = [&](const uint8_t* base, int64_t pitch) __attribute__((always_inline)) {
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base + n0 * pitch), 0, rows * (int)pitch, 0x00020000);
        };
        const auto codes = buffer(w, p.code_pitch), scales = buffer(ws, p.scale_pitch);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int step = 4 * group + s < p.last_step ? 4 * group + s : p.last_step;          // (a row's scales are zeros past its end)
            o.w[s] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(codes, r * (int)p.code_pitch + 16 * g, rows ? step * 64 : 0, 0));
        }
        o.ws = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(scales, r * (int)p.scale_pitch, rows ? group * 16 : 0, 0));
    };
    auto fetch_rows = [&](Rows& o, int group) __attribute__((always_inline)) {
        group = group < p.groups ? group : p.groups - 1;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int64_t m = row0 + (16 * i + r < M ? 16 * i + r : M - 1);      // (rows past the last one make results that are not stored)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int step = 4 * group + s < p.last_step ? 4 * group + s : p.last_step;
                o.a[i][s] = *reinterpret_cast<const v4i*>(p.a + m * p.code_pitch + 16 * g + (int64_t)step * 64);
            }
            o.as[i] = *reinterpret_cast<const v4u*>(p.as + m * p.scale_pitch + (int64_t)group * 16);
        }
    };

    Weights next, after;                 // the next block's (SINGLE: and the one behind it)
    Rows rows;
    if constexpr (kQuantise) {
        // Its group of the rows through LDS, which the sums take over.  (Four rows' loads at once, before the weights', none in a branch that would have one wait for
        // another: lanes past a row's whole runs read its first.)
        const int col = wave * kScaleUnit + 8 * lane, n = p.K - col;
        const X* const x = static_cast<const X*>(p.x) + (int64_t)row0 * p.ldx;
        uint8_t* const mine = lds + wave * M * kFewRow;
        bool fetched = false;
        for (int m0 = 0; m0 < M; m0 += 4) {
            float v[4][8];
            const X* row[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) row[i] = x + (m0 + i < M ? m0 + i : M - 1) * p.ldx;
            Raw8<X> raw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                raw[i] = Raw8<X>{};
                if (p.K >= 8 && m0 + i < M) load_raw<false>(row[i] + (n >= 8 ? col : 0), raw[i]);
            }
            if (!fetched) {
                fetch(next, 0, wave);
                fetch(after, 1, wave);
            }
            fetched = true;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                values_of(raw[i], v[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = n >= 8 ? v[i][e] : 0.0f;
            }
            if (p.K % 8 && n > 0 && n < 8) {                 // the lane that holds a row's end
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
                if (m0 + i >= M) break;
                const uint32_t byte = scale4_of(block_top(v[i]));
                uint8_t* to = mine + (m0 + i) * kFewRow;
                *reinterpret_cast<uint32_t*>(to + 4 * lane) = codes4_of(v[i], byte);
                if ((lane & 3) == 0) to[256 + 16 + (lane >> 2)] = (uint8_t)byte;
            }
        }
        wavefront_lds_fence();
        const uint8_t* from = mine + (r < M ? r : 0) * kFewRow;
        rows.as[0] = *reinterpret_cast<const v4u*>(from + 256 + 16);
#pragma unroll
        for (int s = 0; s < 4; ++s) rows.a[0][s] = *reinterpret_cast<const v4i*>(from + s * 64 + 16 * g);
        __syncthreads();
    } else {
        fetch_rows(rows, wave);
        fetch(next, 0, wave);
        if constexpr (SINGLE) fetch(after, 1, wave);
    }

    for (int block = 0; block < blocks; ++block) {
        v4f acc[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[i] = v4f{};
        const auto multiply = [&](const Weights& now) __attribute__((always_inline)) {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const v8i wv = __builtin_shufflevector(now.w[s], now.w[s], 0, 1, 2, 3, -1, -1, -1, -1);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const v8i av = __builtin_shufflevector(rows.a[i][s], rows.a[i][s], 0, 1, 2, 3, -1, -1, -1, -1);
                    acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, av, acc[i], 4, 4, 0, now.ws[s] >> (8 * g), 0, rows.as[i][s] >> (8 * g));
                }
            }
        };
        if constexpr (SINGLE) {
            const Weights now = next;
            next = after;
            fetch(after, block + 2, wave);
            if (wave < p.groups) multiply(now);
        } else {
            for (int group = wave; group < p.groups; group += WAVES) {
                const Weights now = next;
                const Rows these = rows;
                const bool last = group + WAVES >= p.groups;
                Rows more;
                fetch_rows(more, last ? wave : group + WAVES);
                fetch(next, last ? block + 1 : block, last ? wave : group + WAVES);
                rows = these;
                multiply(now);
                rows = more;
            }
        }
        // ---- the wavefronts' sums, in one of two places by turns: a barrier a block is enough
        v4f* const sums = reinterpret_cast<v4f*>(lds) + (block & 1) * (WAVES * MT * 64);
#pragma unroll
        for (int i = 0; i < MT; ++i) sums[(wave * MT + i) * 64 + lane] = acc[i];
        __syncthreads();
        for (int t = threadIdx.x; t < MT * 256; t += WAVES * 64) {
            const int i = t >> 8, from = (t >> 2) & 63, e = t & 3, m = 16 * i + (from & 15), n = (block0 + block) * kFewColumns + 4 * (from >> 4) + e;
            if (m >= M || n >= p.N) continue;
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) s += reinterpret_cast<const float*>(sums)[((k * MT + i) * 64 + from) * 4 + e];
            const int64_t row = row0 + m;
            s = p.epilogue.template apply<O>(s + (p.bias ? p.bias[(int64_t)expert * p.N + n] : 0.0f));
            y[row * p.ldy + n] = (O)(p.epilogue.residual ? s + (float)static_cast<const O*>(p.epilogue.residual)[row * p.epilogue.ldr + n] : s);
        }
    }
#endif
}
#endif

template <int WAVES, int MT>
inline size_t experts_few_lds_bytes(int rows, bool quantise) {
    const size_t sums = 2 * (size_t)WAVES * MT * 64 * 16, coded = quantise ? (size_t)WAVES * rows * kFewRow : 0;
    return sums > coded ? sums : coded;
}

}  // namespace mx
}  // namespace sparq
