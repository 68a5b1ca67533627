// The gradients' kernels by tile, types and direction; a translation unit each (sparq_mx_grad_*.hip).
#pragma once
#include <type_traits>

#include "sparq_mx_grad_wide_kernel.h"

namespace sparq {
namespace mx {

// Implemented in sparq_mx_grad_{dx,dw}_{bf16,f16,f32}.hip.
#define SPARQ_MX_GRAD_DECLARE(NAME) sparq_status NAME(const GradParams& p, int parts, int tile, void* out, int out_type, hipStream_t stream);
SPARQ_MX_GRAD_DECLARE(launch_grad_dx_bf16)
SPARQ_MX_GRAD_DECLARE(launch_grad_dx_f16)
SPARQ_MX_GRAD_DECLARE(launch_grad_dx_f32)
SPARQ_MX_GRAD_DECLARE(launch_grad_dw_bf16)
SPARQ_MX_GRAD_DECLARE(launch_grad_dw_f16)
SPARQ_MX_GRAD_DECLARE(launch_grad_dw_f32)

inline sparq_status launch_grad(const GradParams& p, int parts, int tile, int dy_type, bool dw, void* out, int out_type, hipStream_t stream) {
    const auto f = dy_type == SPARQ_MX_BF16  ? (dw ? launch_grad_dw_bf16 : launch_grad_dx_bf16)
                   : dy_type == SPARQ_MX_F16 ? (dw ? launch_grad_dw_f16 : launch_grad_dx_f16)
                                             : (dw ? launch_grad_dw_f32 : launch_grad_dx_f32);
    return f(p, parts, tile, out, out_type, stream);
}

template <class O, class F>
sparq_status launch_grad_kernel(F* kernel, int lds_bytes, std::atomic<bool> (&allowed)[kMaxDevices], const GradParams& p, int parts, void* out,
                                hipStream_t stream) {
    const int slot = current_device_slot();                  // the attribute is set once per device (twice at worst)
    if (!allowed[slot].load(std::memory_order_relaxed) || slot == kMaxDevices - 1) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes) != hipSuccess)
            return SPARQ_ELAUNCH;
        allowed[slot].store(true, std::memory_order_relaxed);
    }
    constexpr int kColumns = ColumnSums<float, kGradThreads>::kColumns;
    const int64_t sums = p.slabs * ((p.J + kColumns - 1) / kColumns);
    kernel<<<dim3((unsigned)(p.tiles_j * (int64_t)p.tiles_k + sums), parts), kGradThreads, lds_bytes, stream>>>(static_cast<O*>(out), p);
    return launch_status();
}
template <class T, bool DW>
sparq_status launch_grad_types(const GradParams& p, int parts, int tile, void* out, int out_type, hipStream_t stream) {
    sparq_status s = SPARQ_OK;
    with_type(out_type, [&](auto o) {
        typedef decltype(o) O;
        static std::atomic<bool> allowed[3][kMaxDevices];
        if constexpr (std::is_same_v<T, __bf16>) {
            if (tile == 256) {
                s = launch_grad_kernel<O>(grad_wide_kernel<T, O, DW, 256>, kWideLds<T, 256>, allowed[0], p, parts, out, stream);
                return;
            }
        }
        s = tile == 128 ? launch_grad_kernel<O>(grad_wide_kernel<T, O, DW, 128>, kWideLds<T, 128>, allowed[1], p, parts, out, stream)
                        : launch_grad_kernel<O>(grad_wide_kernel<T, O, DW, 64>, kWideLds<T, 64>, allowed[2], p, parts, out, stream);
    });
    return s;
}

}  // namespace mx
}  // namespace sparq
