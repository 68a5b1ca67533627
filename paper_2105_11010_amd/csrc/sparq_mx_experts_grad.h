// The experts' gradients: the kernel of sparq_mx_grad_wide_kernel.h with rows of several experts; a translation unit for each type of dy and direction.
#pragma once
#include "sparq_mx_grad.h"

namespace sparq {
namespace mx {

struct ExpertGradParams : GradParams {
    const ExpertTile* table;             // dx: tiles of rows (NULL: by the offsets, at most 64 experts)
    const int32_t* offsets;
    int32_t experts;
    int64_t rows;                        // of dy and of X or dx
    int32_t margin;                      // dw: an expert's last rows that are not read in whole runs

#if defined(__HIP_DEVICE_COMPILE__)
    // dw: what is the workgroup's own of the call, its expert's rows.
    template <class T>
    __device__ __forceinline__ void own_rows(GradParams& p) const {
        ConstantInt* const at = (ConstantInt*)(offsets + blockIdx.y);
        const int most = (int)rows, a = at[0], b = at[1], first = a < 0 ? 0 : a > most ? most : a, end = b > most ? most : b;
        p.R = end > first ? end - first : 0;
        p.dy = static_cast<const T*>(dy) + first * lddy;
        p.codes = codes + first * code_pitch;
        p.scales = scales + first * scale_pitch;
        p.steps_per_part = (int)((p.R + kGradStep - 1) / kGradStep);
        const int64_t whole = p.R - margin;
        p.s_whole = whole > 0 && s_whole > 0 ? whole / kGradStep : 0;
    }
    // dx: the workgroup's tile, its first row and column (in tiles); false: there are fewer tiles.
    template <int TILE>
    __device__ __forceinline__ bool own_tile(GradParams& p, int64_t& j0, uint32_t& tk) const {
        LaneTiles lanes = {};
        if (!table) lanes = tiles_of_lanes(offsets, experts, rows, TILE);
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
