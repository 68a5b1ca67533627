// The product of 4-bit operands (include/sparq_mx.h).
#include "sparq_mx_few.h"
#include "sparq_mx_gemm_kernel.h"

namespace sparq {
namespace mx {

struct GemmPlan {
    int tile;                // 256, 128 or 64: results a workgroup makes along either side; 0: few rows, a kernel of their own
    int parts;               // of the reduction
    size_t bytes;            // of partial results
};
static GemmPlan gemm_plan(int64_t M, int N, int K) {
    GemmPlan p = {};
    // Few rows: the kernel that reads the weights at memory's pace, while its rereading of A is no longer than that (us, it -> 64 x 64 tiles:
    // 17 x 4096 x 4096 4.7 -> 6.4, 32 x 4096 x 4096 5.6 -> 7.0, 48 x 4096 x 4096 7.0 -> 6.6, 64 x 4096 x 4096 8.2 -> 6.9, 32 x 8192 x 8192 16 -> 12.5).
    if (M <= 16 || (M <= kFewMost && M * N * K <= 5ll << 27)) return p;
    const auto tiles = [&](int t) { return ((M + t - 1) / t) * ((N + t - 1) / t); };
    // The larger tiles, one a CU at a time, unless they leave CUs without (us, 256 x 256 -> 128 x 128: 4096^3 47 -> 54, 3584^3 37 -> 47, 3000^3
    // 30 -> 30, 4096 x 2048 x 4096 34 -> 28, 2900 x 3700 x 2500 30 -> 27, 2048^3 18 -> 10; 128 x 128, two a CU, -> 64 x 64, three: 2048^3 9.4 -> 13,
    // 600 x 3000 x 8192 21.8 -> 23.6, 512 x 3000 x 2048 7.8 -> 7.3, 200 x 3000 x 3000 9.0 -> 6.1, 515 x 771 x 577 5.9 -> 4.5): what a CU can load of
    // codes bounds each of them.
    p.tile = tiles(256) >= 192 ? 256 : tiles(128) >= 112 ? 128 : 64;
    // Few tiles of a long reduction are divided; shorter ones, or more of them, are over before the parts would be joined (us, whole -> in
    // parts: 70 x 300 x 16000 17.2 -> 9.6, 65 x 1000 x 8192 10.2 -> 9.3; with up to 128 tiles of 32 steps: 100 x 500 x 4096 6.7 -> 8.7).
    const int64_t n = tiles(p.tile), steps = (K + kCodeUnit - 1) / kCodeUnit, most = steps / 16;
    p.parts = n <= 64 && steps >= 64 ? (int)(128 / n < most ? 128 / n : most) : 1;
    p.bytes = p.parts > 1 ? (size_t)round_up(p.parts * M * N * 4, 256) : 0;
    return p;
}

// As many tiles, with their parts, as the kernel counts
static bool countable(const GemmPlan& p, int64_t M, int64_t N) {
    const int t = p.tile;
    return t == 0 || (M + t - 1) / t * ((N + t - 1) / t) * p.parts < (1ll << 31);
}

template <class O, int TILE>
static sparq_status launch_tile(const GemmParams& p, void* y, hipStream_t stream) {
    const auto kernel = gemm_kernel<O, TILE, TILE>;
    constexpr int lds_bytes = kGemmLds<TILE>, per_cu = 160 * 1024 / lds_bytes;
    static_assert(per_cu >= 1, "LDS of a CU");
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

static sparq_status gemm(const void* a, const void* as, const void* w, const void* ws, const float* bias, void* y, int type, int64_t ldy,
                         int64_t M, int N, int K, const GemmPlan& plan, void* workspace, hipStream_t stream) {
    const int t = plan.tile;
    if (t == 0) {
        const FewParams f = {nullptr, static_cast<const uint8_t*>(a), static_cast<const uint8_t*>(as), static_cast<const uint8_t*>(w),
                             static_cast<const uint8_t*>(ws), bias, 0, ldy, code_pitch(K, 4), scale_pitch(K), (int)M, N, K,
                             (K + kScaleUnit - 1) / kScaleUnit, (K + kCodeUnit - 1) / kCodeUnit - 1};
        return launch_few_rows(f, 0, y, type, stream);
    }
    const int64_t tiles_m = (M + t - 1) / t, tiles_n = (N + t - 1) / t;
    const bool parted = plan.parts > 1;
    GemmParams p = {};
    p.a = static_cast<const uint8_t*>(a);
    p.as = static_cast<const uint8_t*>(as);
    p.w = static_cast<const uint8_t*>(w);
    p.ws = static_cast<const uint8_t*>(ws);
    p.bias = parted ? nullptr : bias;
    p.M = M;
    p.N = N;
    p.ldy = parted ? N : ldy;
    p.part_stride = parted ? M * N : 0;
    p.code_pitch = (uint32_t)code_pitch(K, 4);
    p.scale_pitch = (uint32_t)scale_pitch(K);
    p.tiles_m = (uint32_t)tiles_m;
    p.tiles_n = (uint32_t)tiles_n;
    p.steps = (int)round_up((K + kCodeUnit - 1) / kCodeUnit, 4);
    p.steps_per_part = (int)round_up((p.steps + plan.parts - 1) / plan.parts, 4);
    const int parts = (p.steps + p.steps_per_part - 1) / p.steps_per_part;       // (as the plan has it, or fewer)
    p.items = (uint32_t)(tiles_m * tiles_n * parts);
    sparq_status s = SPARQ_OK;
    with_type(parted ? SPARQ_MX_F32 : type, [&](auto o) {
        typedef decltype(o) O;
        void* to = parted ? workspace : y;
        s = t == 256 ? launch_tile<O, 256>(p, to, stream) : t == 128 ? launch_tile<O, 128>(p, to, stream) : launch_tile<O, 64>(p, to, stream);
    });
    if (s != SPARQ_OK || !parted) return s;
    return launch_join(static_cast<const float*>(workspace), bias, y, type, M, N, ldy, parts, stream);
}

static bool gemm_sizes_ok(int64_t M, int64_t N, int64_t K) { return sizes_ok(M, K) && N >= 1 && N <= kMaxK && M < (1ll << 40) && K <= kGemmMaxK; }

}  // namespace mx
}  // namespace sparq

using namespace sparq;
using namespace sparq::mx;

extern "C" size_t sparq_mx_gemm_workspace_bytes(int64_t M, int32_t N, int32_t K) {
    return gemm_sizes_ok(M, N, K) && M > 0 ? gemm_plan(M, N, K).bytes : 0;
}

extern "C" sparq_status sparq_mx_gemm(const void* a_codes, const void* a_scales, const void* w_codes, const void* w_scales,
                                      const float* bias, void* y, int32_t type, int64_t ldy, int64_t M, int32_t N, int32_t K,
                                      void* workspace, size_t workspace_bytes, void* stream) {
    if (!gemm_sizes_ok(M, N, K) || !type_valid(type)) return SPARQ_EINVAL;
    if (M == 0) return SPARQ_OK;
    if (!coded_ok(a_codes, a_scales) || !coded_ok(w_codes, w_scales) || !aligned(bias, 4)) return SPARQ_EINVAL;
    if (!tensor_ok(y, type, ldy, N) || !extent_ok(M, ldy) || !extent_ok(M, K)) return SPARQ_EINVAL;
    const GemmPlan plan = gemm_plan(M, N, K);
    if (plan.bytes && (!workspace || !aligned(workspace, 256))) return SPARQ_EINVAL;
    if (workspace_bytes < plan.bytes) return SPARQ_EWORKSPACE;
    if (!countable(plan, M, N)) return SPARQ_EUNSUPPORTED;
    return gemm(a_codes, a_scales, w_codes, w_scales, bias, y, type, ldy, M, N, K, plan, workspace, static_cast<hipStream_t>(stream));
}

// Whether the product quantises its rows itself: what that saves is a launch, about 3 us, and what it costs is every workgroup doing it
// again (us, itself -> before it: 8 x 4096 x 4096 6.1 -> 6.9, 16 x 4096 x 4096 8.1 -> 7.1, 1 x 8192 x 8192 9.4 -> 10.8, 8 x 8192 x 8192
// 15.2 -> 12.5).
static bool quantised_on_the_way(int64_t M, int N, int K) { return M <= kFewRows && M * N * K <= 1 << 27; }
static size_t coded_bytes(int64_t M, int N, int K) {
    if (quantised_on_the_way(M, N, K)) return 0;
    return (size_t)(round_up(M * code_pitch(K, 4), 256) + round_up(M * scale_pitch(K), 256));
}

extern "C" size_t sparq_mx_linear_workspace_bytes(int64_t M, int32_t N, int32_t K) {
    return gemm_sizes_ok(M, N, K) && M > 0 ? coded_bytes(M, N, K) + gemm_plan(M, N, K).bytes : 0;
}

extern "C" sparq_status sparq_mx_linear(const void* x, int32_t x_type, int64_t ldx, const void* w_codes, const void* w_scales,
                                        const float* bias, void* y, int32_t y_type, int64_t ldy, int64_t M, int32_t N, int32_t K,
                                        void* workspace, size_t workspace_bytes, void* stream) {
    if (!gemm_sizes_ok(M, N, K) || !type_valid(x_type) || !type_valid(y_type)) return SPARQ_EINVAL;
    if (M == 0) return SPARQ_OK;
    if (!coded_ok(w_codes, w_scales) || !aligned(bias, 4)) return SPARQ_EINVAL;
    if (!tensor_ok(x, x_type, ldx, K) || !extent_ok(M, ldx) || !tensor_ok(y, y_type, ldy, N) || !extent_ok(M, ldy) || !extent_ok(M, K))
        return SPARQ_EINVAL;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (quantised_on_the_way(M, N, K)) {
        const FewParams f = {x, nullptr, nullptr, static_cast<const uint8_t*>(w_codes), static_cast<const uint8_t*>(w_scales), bias, ldx, ldy,
                             code_pitch(K, 4), scale_pitch(K), (int)M, N, K, (K + kScaleUnit - 1) / kScaleUnit, (K + kCodeUnit - 1) / kCodeUnit - 1};
        return launch_few_rows(f, x_type, y, y_type, s);
    }
    const GemmPlan plan = gemm_plan(M, N, K);
    const size_t coded = coded_bytes(M, N, K);
    if (!workspace || !aligned(workspace, 256)) return SPARQ_EINVAL;
    if (workspace_bytes < coded + plan.bytes) return SPARQ_EWORKSPACE;
    if (!countable(plan, M, N)) return SPARQ_EUNSUPPORTED;
    uint8_t *codes = static_cast<uint8_t*>(workspace), *scales = codes + round_up(M * code_pitch(K, 4), 256);
    const sparq_status q = launch_quantize(x, x_type, ldx, M, K, codes, scales, nullptr, nullptr, s);
    if (q != SPARQ_OK) return q;
    return gemm(codes, scales, w_codes, w_scales, bias, y, y_type, ldy, M, N, K, plan, codes + coded, s);
}
