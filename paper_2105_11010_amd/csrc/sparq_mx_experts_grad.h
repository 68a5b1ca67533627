// The experts' gradients: the kernel of sparq_mx_grad_wide_kernel.h with rows of several experts; a translation unit for each type of dy and direction.
// 16384 x 2048 x 2048 to 8 experts, bf16, on the same tensors again and on four sets in turn: dx 112-116 and 118 us of even ones, 137 and 140 of uneven ones (two launches,
// 114-128 and 28), dw 141-144 and 150, 143 and 154 (0.9-1.24 PF; the dense kernels 1.07-1.33).
#pragma once
#include "sparq_mx_grad.h"

namespace sparq {
namespace mx {

// (of 64 finding them costs what it gains: 16384 rows to 512 x 512 each 35 -> 40 us; 16384 to 8 of 2048 x 2048, uneven, 163 -> 146)
constexpr int kLongestFirst = 16;

struct ExpertGradParams : GradParams {
    const ExpertTile* table;             // dx: tiles of rows (NULL: by the offsets, at most 64 experts)
    const int32_t* offsets;
    int32_t experts;
    int64_t rows;                        // of dy and of X or dx
    int32_t whole;                       // dx, without a table: n > 0: each expert's first whole n rows alone; n < 0: what is left behind whole -n rows; 0: all rows
    int32_t margin;                      // dw: dy's last rows, which are not read in whole runs (or all of them)

#if defined(__HIP_DEVICE_COMPILE__)
    // dw: what is the workgroup's own of the call, the rows and results of an expert.  Of a few experts those with the most rows come first: the tiles of a
    // launch's last round are its shortest ones then.
    template <class T, class O>
    __device__ __forceinline__ O* own_rows(GradParams& p, O* out) const {
        uint32_t expert = blockIdx.y;
        if (experts <= kLongestFirst) {
            const int lane = threadIdx.x & 63;
            int first = 0, n = -1;
            if (lane < experts) expert_rows(offsets, lane, rows, first, n);
            uint32_t before = 0;
            for (int e = 0; e < experts; ++e) {
                const int other = __builtin_amdgcn_readlane(n, e);
                before += other > n || (other == n && e < lane) ? 1 : 0;
            }
            expert = (uint32_t)__builtin_ctzll(__ballot(lane < experts && before == blockIdx.y) | 1ull << 63);
        }
        ConstantInt* const at = (ConstantInt*)(offsets + expert);
        const int most = (int)rows, a = at[0], b = at[1], first = a < 0 ? 0 : a > most ? most : a, end = b > most ? most : b;
        p.R = end > first ? end - first : 0;
        p.dy = static_cast<const T*>(dy) + first * lddy;
        p.codes = codes + first * code_pitch;
        p.scales = scales + first * scale_pitch;
        p.steps_per_part = (int)((p.R + kGradStep - 1) / kGradStep);
        const int64_t most_fast = rows - margin - first;
        p.slab = p.R < most_fast ? p.R : most_fast > 0 ? most_fast : 0;
        if (kParts<T> > 1) p.slab = p.slab / kGradStep * kGradStep;          // (the others' last step may have fewer rows)
        p.s_whole = (p.slab + kGradStep - 1) / kGradStep;
        if (column_sums) p.column_sums = column_sums + (int64_t)expert * J;
        return out + (int64_t)expert * J * ldo;
    }
    // dw: as many of the expert's rows as are read in whole runs, those whose runs end inside dy (own_rows), and what is left behind them.
    __device__ __forceinline__ int fast_rows(const GradParams& p) const { return (int)p.slab; }
    template <class T>
    __device__ __forceinline__ void leave_fast(GradParams& p) const {
        const int64_t n = p.slab;
        p.dy = static_cast<const T*>(p.dy) + n * lddy;
        p.codes += n * code_pitch;
        p.scales += n * scale_pitch;
        p.R -= n;
        p.steps_per_part = (int)((p.R + kGradStep - 1) / kGradStep);
    }
    // dx: the workgroup's tile, its first row and column (in tiles); false: there are fewer tiles.
    template <int TILE>
    __device__ __forceinline__ bool own_tile(GradParams& p, int64_t& j0, uint32_t& tk) const {
        LaneTiles lanes = {};
        if (!table) lanes = tiles_of_lanes(offsets, experts, rows, TILE, whole);
        const uint32_t tiles = (uint32_t)(table ? tile_count(table) : tile_count(lanes));
        if (blockIdx.x >= tiles * (uint32_t)tiles_k) return false;
        uint32_t tj;
        tile_of(blockIdx.x, tiles, tiles_k, tj, tk);
        const ExpertTile t = table ? expert_tile(table, tj) : expert_tile(lanes, TILE, tj);
        j0 = t.row;
        p.J = t.row + t.rows;
        p.codes = codes + (int64_t)t.expert * R * code_pitch;
        p.scales = scales + (int64_t)t.expert * R * scale_pitch;
        return true;
    }
#endif
};

// Implemented in sparq_mx_experts_{dx,dw}_{bf16,f16,f32}.hip.
#define SPARQ_MX_EXPERTS_GRAD_DECLARE(NAME) sparq_status NAME(const ExpertGradParams& p, dim3 grid, int tile, void* out, bool f32, hipStream_t stream);
SPARQ_MX_EXPERTS_GRAD_DECLARE(launch_experts_dx_bf16)
SPARQ_MX_EXPERTS_GRAD_DECLARE(launch_experts_dx_f16)
SPARQ_MX_EXPERTS_GRAD_DECLARE(launch_experts_dx_f32)
SPARQ_MX_EXPERTS_GRAD_DECLARE(launch_experts_dw_bf16)
SPARQ_MX_EXPERTS_GRAD_DECLARE(launch_experts_dw_f16)
SPARQ_MX_EXPERTS_GRAD_DECLARE(launch_experts_dw_f32)

template <class O, class F>
sparq_status launch_experts_grad_kernel(F* kernel, int lds_bytes, std::atomic<bool> (&allowed)[kMaxDevices], const ExpertGradParams& p, dim3 grid, void* out,
                                        hipStream_t stream) {
    const int slot = current_device_slot();                  // the attribute is set once per device (twice at worst)
    if (!allowed[slot].load(std::memory_order_relaxed) || slot == kMaxDevices - 1) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes) != hipSuccess)
            return SPARQ_ELAUNCH;
        allowed[slot].store(true, std::memory_order_relaxed);
    }
    kernel<<<grid, kGradThreads, lds_bytes, stream>>>(static_cast<O*>(out), p);
    return launch_status();
}
template <class T, class O, bool DW>
sparq_status launch_experts_grad_types(const ExpertGradParams& p, dim3 grid, int tile, void* out, hipStream_t stream) {
    static std::atomic<bool> allowed[3][kMaxDevices];
    if constexpr (std::is_same_v<T, __bf16>)
        if (tile == 256) return launch_experts_grad_kernel<O>(grad_wide_kernel<T, O, DW, 256, ExpertGradParams>, kWideLds<T, 256>, allowed[0], p, grid, out, stream);
    return tile == 128 ? launch_experts_grad_kernel<O>(grad_wide_kernel<T, O, DW, 128, ExpertGradParams>, kWideLds<T, 128>, allowed[1], p, grid, out, stream)
                       : launch_experts_grad_kernel<O>(grad_wide_kernel<T, O, DW, 64, ExpertGradParams>, kWideLds<T, 64>, allowed[2], p, grid, out, stream);
}
// f32: results of fp32, else of dy's type
template <class T, bool DW>
sparq_status launch_experts_grad(const ExpertGradParams& p, dim3 grid, int tile, void* out, bool f32, hipStream_t stream) {
    return f32 ? launch_experts_grad_types<T, float, DW>(p, grid, tile, out, stream) : launch_experts_grad_types<T, T, DW>(p, grid, tile, out, stream);
}

}  // namespace mx
}  // namespace sparq
