// The experts' products and a layer with an epilogue: entry points, tiles of rows, the join of a divided reduction (include/sparq_mx_experts.h).
#include "sparq_mx_experts_gemm.h"
#include "sparq_mx_experts_plan.h"

namespace sparq {
namespace mx {

// ---- tiles of rows ---------------------------------------------------------------------
// Each expert's rows in tiles of their own.
__global__ __launch_bounds__(kTableThreads) void tiles_kernel(const int32_t* __restrict__ offsets, int experts, int64_t rows, int tile, int most,
                                                              ExpertTile* __restrict__ table) {
    __shared__ int64_t sums[kTableThreads / 64];
    write_tiles(offsets, experts, rows, tile, most, table, sums);
}
sparq_status launch_tiles(const int32_t* offsets, int experts, int64_t rows, int tile, void* table, hipStream_t stream) {
    tiles_kernel<<<1, kTableThreads, 0, stream>>>(offsets, experts, rows, tile, (int)most_tiles(rows, experts, tile), static_cast<ExpertTile*>(table));
    return launch_status();
}

// ---- parts of a divided reduction, and the epilogue of their sum -------------------------
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
template <class O>
__global__ __launch_bounds__(kThreads) void finish_kernel(const float* __restrict__ partial, const float* __restrict__ bias, O* __restrict__ y, int64_t ldy,
                                                          int64_t M, int N, int parts, int chunks, uint32_t items, const Epilogue epilogue) {
    const uint32_t item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= items) return;
    const int64_t row = item / (uint32_t)chunks;
    const int col = (int)(item - row * chunks) * kScaleUnit + 8 * (threadIdx.x & 63), n = N - col;
    float z[8] = {};
    for (int i = 0; i < parts; ++i) {
        float v[8];
        load_upto8(partial + (i * M + row) * N + col, n, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] += v[e];
    }
    if (bias) {
        float b[8];
        load_upto8(bias + col, n, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] += b[e];
    }
    epilogue.finish<O>(z, y, ldy, row, col, n, true);
}

struct Call {
    const void* x;           // rows to be quantised on the way (few rows), or
    int x_type;
    int64_t ldx;
    const void *a, *as;      // codes and scales
    const int32_t* offsets;
    int experts;
    const void *w, *ws;
    const float* bias;
    Epilogue epilogue;
    void* y;
    int type;
    int64_t ldy, M;
    int N, K;
};

static sparq_status launch_tiles_of(const ExpertGemmParams& p, int tile, void* y, int type, hipStream_t stream) {
    return (type == SPARQ_MX_F32 ? launch_experts_tiles_f32 : type == SPARQ_MX_F16 ? launch_experts_tiles_f16 : launch_experts_tiles_bf16)(p, tile, y, stream);
}

static sparq_status product(const Call& c, const ExpertsPlan& plan, void* workspace, hipStream_t stream) {
    if (plan.tile == 0) {
        ExpertFewParams f = {};
        f.x = c.x;
        f.a = static_cast<const uint8_t*>(c.a);
        f.as = static_cast<const uint8_t*>(c.as);
        f.w = static_cast<const uint8_t*>(c.w);
        f.ws = static_cast<const uint8_t*>(c.ws);
        f.bias = c.bias;
        f.offsets = c.offsets;
        f.ldx = c.ldx;
        f.ldy = c.ldy;
        f.code_pitch = code_pitch(c.K, 4);
        f.scale_pitch = scale_pitch(c.K);
        f.M = c.M;
        f.N = c.N;
        f.K = c.K;
        f.groups = (c.K + kScaleUnit - 1) / kScaleUnit;
        f.last_step = (c.K + kCodeUnit - 1) / kCodeUnit - 1;
        f.experts = c.experts;
        f.blocks = plan.blocks;
        f.epilogue = c.epilogue;
        return (c.type == SPARQ_MX_F32 ? launch_experts_few_f32 : c.type == SPARQ_MX_F16 ? launch_experts_few_f16 : launch_experts_few_bf16)(
            f, c.x_type, plan.fragments, plan.pieces, c.y, stream);
    }
    const int t = plan.tile;
    const bool parted = plan.parts > 1;
    const int64_t tiles_m = c.offsets ? most_tiles(c.M, c.experts, t) : (c.M + t - 1) / t, tiles_n = (c.N + t - 1) / t;
    ExpertGemmParams p = {};
    p.a = static_cast<const uint8_t*>(c.a);
    p.as = static_cast<const uint8_t*>(c.as);
    p.w = static_cast<const uint8_t*>(c.w);
    p.ws = static_cast<const uint8_t*>(c.ws);
    p.bias = parted ? nullptr : c.bias;
    p.M = c.M;
    p.N = c.N;
    p.ldy = parted ? c.N : c.ldy;
    p.part_stride = parted ? c.M * c.N : 0;
    p.code_pitch = (uint32_t)code_pitch(c.K, 4);
    p.scale_pitch = (uint32_t)scale_pitch(c.K);
    p.tiles_m = (uint32_t)tiles_m;
    p.tiles_n = (uint32_t)tiles_n;
    p.steps = (int)round_up((c.K + kCodeUnit - 1) / kCodeUnit, 4);
    p.steps_per_part = (int)round_up((p.steps + plan.parts - 1) / plan.parts, 4);
    const int parts = (p.steps + p.steps_per_part - 1) / p.steps_per_part;       // (as the plan has it, or fewer)
    p.items = (uint32_t)(tiles_m * tiles_n * parts);
    if (parted) p.epilogue.function = SPARQ_MX_NONE;
    else p.epilogue = c.epilogue;
    p.offsets = c.offsets;
    p.experts = c.experts;
    if (plan.table_bytes) {
        p.table = static_cast<const ExpertTile*>(workspace);
        const sparq_status s = launch_tiles(c.offsets, c.experts, c.M, t, workspace, stream);
        if (s != SPARQ_OK) return s;
    }
    const sparq_status s = launch_tiles_of(p, t, parted ? workspace : c.y, parted ? SPARQ_MX_F32 : c.type, stream);
    if (s != SPARQ_OK || !parted) return s;
    const int chunks = (c.N + kScaleUnit - 1) / kScaleUnit;
    with_type(c.type, [&](auto o) {
        typedef decltype(o) O;
        const uint32_t items = (uint32_t)(c.M * chunks);
        finish_kernel<O><<<(items + kWaves - 1) / kWaves, kThreads, 0, stream>>>(static_cast<const float*>(workspace), c.bias, static_cast<O*>(c.y), c.ldy, c.M,
                                                                                c.N, parts, chunks, items, c.epilogue);
    });
    return launch_status();
}

// As many tiles, with their parts, as the kernels count
static bool countable(const ExpertsPlan& p, int64_t M, int64_t N, int experts) {
    if (M >= 1ll << 31 || experts > SPARQ_MX_EXPERTS_MOST || (int64_t)experts * N >= 1ll << 31) return false;
    if (p.tile == 0) return true;                            // (at most 1792 pieces, and 8 blocks a workgroup of many)
    const int t = p.tile;
    return (M / t + 1 + experts) * ((N + t - 1) / t) * p.parts < (1ll << 31);
}

static bool experts_sizes_ok(int64_t M, int64_t N, int64_t K, int64_t experts) {
    return sizes_ok(M, K) && N >= 1 && N <= kMaxK && M < (1ll << 40) && K <= kGemmMaxK && experts_ok((int)experts);
}
static bool epilogue_ok(int function, const void* residual, int64_t ldr, int type, const void* kept_codes, const void* kept_scales, int64_t M, int N) {
    if (function != SPARQ_MX_NONE && function != SPARQ_MX_SILU && function != SPARQ_MX_GELU) return false;
    if (residual && (!tensor_ok(residual, type, ldr, N) || !extent_ok(M, ldr))) return false;
    return coded_ok_or_none(kept_codes, kept_scales) && extent_ok(M, N);
}
static Epilogue epilogue_of(int function, const void* residual, int64_t ldr, void* kept_codes, void* kept_scales, int N) {
    return {residual, static_cast<uint8_t*>(kept_codes), static_cast<uint8_t*>(kept_scales), ldr, code_pitch(N, 8), scale_pitch(N), function,
            (int)round_up(N, kCodeUnit)};
}

static size_t coded_bytes(int64_t M, int K) { return (size_t)(round_up(M * code_pitch(K, 4), 256) + round_up(M * scale_pitch(K), 256)); }

}  // namespace mx
}  // namespace sparq

using namespace sparq;
using namespace sparq::mx;

extern "C" size_t sparq_mx_experts_gemm_workspace_bytes(int64_t M, int32_t N, int32_t K, int32_t experts) {
    return experts_sizes_ok(M, N, K, experts) && M > 0 ? experts_bytes(M, N, K, experts) : 0;
}

extern "C" sparq_status sparq_mx_experts_gemm(const void* a_codes, const void* a_scales, const int32_t* offsets, int32_t experts, const void* w_codes,
                                              const void* w_scales, const float* bias, int32_t function, const void* residual, int64_t ldr, void* y,
                                              int32_t type, int64_t ldy, void* kept_codes, void* kept_scales, int64_t M, int32_t N, int32_t K,
                                              void* workspace, size_t workspace_bytes, void* stream) {
    if (!experts_sizes_ok(M, N, K, experts) || !type_valid(type)) return SPARQ_EINVAL;
    if ((!offsets && experts != 1) || !aligned(offsets, 4)) return SPARQ_EINVAL;
    if (M == 0) return SPARQ_OK;
    if (!coded_ok(a_codes, a_scales) || !coded_ok(w_codes, w_scales) || !aligned(bias, 4)) return SPARQ_EINVAL;
    if (!tensor_ok(y, type, ldy, N) || !extent_ok(M, ldy) || !extent_ok(M, K) || !epilogue_ok(function, residual, ldr, type, kept_codes, kept_scales, M, N))
        return SPARQ_EINVAL;
    const ExpertsPlan plan = experts_plan(M, N, K, experts, offsets != nullptr, function, residual != nullptr, kept_codes != nullptr);
    const size_t bytes = plan.table_bytes + plan.partial_bytes;
    if (bytes && (!workspace || !aligned(workspace, 256))) return SPARQ_EINVAL;
    if (workspace_bytes < bytes) return SPARQ_EWORKSPACE;
    if (!countable(plan, M, N, experts)) return SPARQ_EUNSUPPORTED;
    const Call c = {nullptr, 0, 0, a_codes, a_scales, offsets, experts, w_codes, w_scales, bias,
                    epilogue_of(function, residual, ldr, kept_codes, kept_scales, N), y, type, ldy, M, N, K};
    return product(c, plan, workspace, static_cast<hipStream_t>(stream));
}

extern "C" size_t sparq_mx_experts_linear_workspace_bytes(int64_t M, int32_t N, int32_t K, int32_t experts) {
    if (!experts_sizes_ok(M, N, K, experts) || M == 0) return 0;
    return coded_bytes(M, K) + experts_bytes(M, N, K, experts);
}

extern "C" sparq_status sparq_mx_experts_linear(const void* x, int32_t x_type, int64_t ldx, const int32_t* offsets, int32_t experts, const void* w_codes,
                                                const void* w_scales, const float* bias, int32_t function, const void* residual, int64_t ldr, void* y,
                                                int32_t y_type, int64_t ldy, void* kept_codes, void* kept_scales, int64_t M, int32_t N, int32_t K,
                                                void* workspace, size_t workspace_bytes, void* stream) {
    if (!experts_sizes_ok(M, N, K, experts) || !type_valid(x_type) || !type_valid(y_type)) return SPARQ_EINVAL;
    if ((!offsets && experts != 1) || !aligned(offsets, 4)) return SPARQ_EINVAL;
    if (M == 0) return SPARQ_OK;
    if (!tensor_ok(x, x_type, ldx, K) || !extent_ok(M, ldx) || !coded_ok(w_codes, w_scales) || !aligned(bias, 4)) return SPARQ_EINVAL;
    if (!tensor_ok(y, y_type, ldy, N) || !extent_ok(M, ldy) || !extent_ok(M, K) || !epilogue_ok(function, residual, ldr, y_type, kept_codes, kept_scales, M, N))
        return SPARQ_EINVAL;
    const ExpertsPlan plan = experts_plan(M, N, K, experts, offsets != nullptr, function, residual != nullptr, kept_codes != nullptr);
    const bool on_the_way = quantised_on_the_way(plan, K);
    const size_t coded = on_the_way ? 0 : coded_bytes(M, K), bytes = coded + plan.table_bytes + plan.partial_bytes;
    if (bytes && (!workspace || !aligned(workspace, 256))) return SPARQ_EINVAL;
    if (workspace_bytes < bytes) return SPARQ_EWORKSPACE;
    if (!countable(plan, M, N, experts)) return SPARQ_EUNSUPPORTED;
    Call c = {x, x_type, ldx, nullptr, nullptr, offsets, experts, w_codes, w_scales, bias,
              epilogue_of(function, residual, ldr, kept_codes, kept_scales, N), y, y_type, ldy, M, N, K};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (on_the_way) return product(c, plan, nullptr, s);
    uint8_t *codes = static_cast<uint8_t*>(workspace), *scales = codes + round_up(M * code_pitch(K, 4), 256);
    const sparq_status q = launch_quantize(x, x_type, ldx, M, K, codes, scales, nullptr, nullptr, s);
    if (q != SPARQ_OK) return q;
    c.x = nullptr;
    c.a = codes;
    c.as = scales;
    return product(c, plan, codes + coded, s);
}
