// The experts' products: the kernel of sparq_mx_gemm_kernel.h with rows of several experts and an epilogue, and the one for few rows.
#pragma once
#include "sparq_mx_epilogue.h"
#include "sparq_mx_experts_few_kernel.h"
#include "sparq_mx_gemm_kernel.h"
#include "sparq_mx_tiles.h"

namespace sparq {
namespace mx {

struct ExpertGemmParams : GemmParams {
    const ExpertTile* table;             // of the rows' tiles, or NULL and the offsets (at most 64 experts and tiles of 128), or both NULL: one expert, all rows
    const int32_t* offsets;
    int32_t experts;
    Epilogue epilogue;
};
// ... of one function: a kernel each, or a tile's end would hold all of them
template <int F>
struct ExpertGemmParamsOf : ExpertGemmParams {
    static constexpr int kFunction = F;
};

// Implemented in sparq_mx_experts_{gemm,few}_{f32,f16,bf16}.hip, by the results' type.
#define SPARQ_MX_EXPERTS_DECLARE(TYPE)                                                                                              \
    sparq_status launch_experts_tiles_##TYPE(const ExpertGemmParams& p, int tile, void* y, hipStream_t stream);                     \
    sparq_status launch_experts_few_##TYPE(const ExpertFewParams& p, int x_type, int fragments, int64_t pieces, void* y, hipStream_t stream);
SPARQ_MX_EXPERTS_DECLARE(f32)
SPARQ_MX_EXPERTS_DECLARE(f16)
SPARQ_MX_EXPERTS_DECLARE(bf16)

template <class O, int TILE, int F>
sparq_status launch_experts_function(const ExpertGemmParams& all, void* y, hipStream_t stream) {
    const ExpertGemmParamsOf<F> p = {all};
    const auto kernel = gemm_kernel<O, TILE, TILE, ExpertGemmParamsOf<F>>;
    constexpr int lds_bytes = kGemmLds<TILE>, per_cu = 160 * 1024 / lds_bytes;
    static std::atomic<bool> allowed[kMaxDevices];           // the attribute is set once per device (twice at worst)
    const int slot = current_device_slot();
    if (!allowed[slot].load(std::memory_order_relaxed) || slot == kMaxDevices - 1) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes) != hipSuccess)
            return SPARQ_ELAUNCH;
        allowed[slot].store(true, std::memory_order_relaxed);
    }
    const uint32_t places = (uint32_t)(device_cu_count() * per_cu);
    kernel<<<p.items < places ? p.items : places, kGemmThreads, lds_bytes, stream>>>(static_cast<O*>(y), p);
    return launch_status();
}
template <class O, int TILE>
sparq_status launch_experts_tile(const ExpertGemmParams& p, void* y, hipStream_t stream) {
    return p.epilogue.function == SPARQ_MX_SILU   ? launch_experts_function<O, TILE, SPARQ_MX_SILU>(p, y, stream)
           : p.epilogue.function == SPARQ_MX_GELU ? launch_experts_function<O, TILE, SPARQ_MX_GELU>(p, y, stream)
                                                  : launch_experts_function<O, TILE, SPARQ_MX_NONE>(p, y, stream);
}
template <class O>
sparq_status launch_experts_tiles(const ExpertGemmParams& p, int tile, void* y, hipStream_t stream) {
    return tile == 256 ? launch_experts_tile<O, 256>(p, y, stream) : tile == 128 ? launch_experts_tile<O, 128>(p, y, stream) : launch_experts_tile<O, 64>(p, y, stream);
}

template <class O, class X, int MT, int WAVES, bool SINGLE>
sparq_status launch_experts_few_kernel(const ExpertFewParams& p, int64_t pieces, void* y, hipStream_t stream) {
    const int rows = p.offsets ? 16 * MT : (int)p.M, blocks = (p.N + kFewColumns - 1) / kFewColumns;
    experts_few_kernel<O, X, MT, WAVES, SINGLE><<<dim3((unsigned)((blocks + p.blocks - 1) / p.blocks), (unsigned)pieces), WAVES * 64,
                                                  experts_few_lds_bytes<WAVES, MT>(rows, p.x != nullptr), stream>>>(static_cast<O*>(y), p);
    return launch_status();
}
template <class O, class X, int MT>
sparq_status launch_experts_waves(const ExpertFewParams& p, int64_t pieces, void* y, hipStream_t stream) {
    if (p.groups <= 4) return launch_experts_few_kernel<O, X, MT, 4, true>(p, pieces, y, stream);
    if (p.groups <= 8) return launch_experts_few_kernel<O, X, MT, 8, true>(p, pieces, y, stream);
    if constexpr (std::is_void_v<X>) return launch_experts_few_kernel<O, X, MT, 8, false>(p, pieces, y, stream);
    return SPARQ_EINVAL;                                     // (nobody asks for it: sparq_mx_experts.hip)
}
// fragments: of 16 rows a workgroup takes
template <class O>
sparq_status launch_experts_few(const ExpertFewParams& p, int x_type, int fragments, int64_t pieces, void* y, hipStream_t stream) {
    sparq_status s = SPARQ_OK;
    if (p.x) with_type(x_type, [&](auto x) { s = launch_experts_waves<O, decltype(x), 1>(p, pieces, y, stream); });
    else if (fragments == 1) s = launch_experts_waves<O, void, 1>(p, pieces, y, stream);
    else if (fragments == 2) s = launch_experts_waves<O, void, 2>(p, pieces, y, stream);
    else if (fragments == 3) s = launch_experts_waves<O, void, 3>(p, pieces, y, stream);
    else s = launch_experts_waves<O, void, 4>(p, pieces, y, stream);
    return s;
}

}  // namespace mx
}  // namespace sparq
