// The experts' products, backward: entry points (include/sparq_mx_experts.h).
#include "sparq_mx_experts_grad.h"
#include "sparq_mx_experts_plan.h"

namespace sparq {
namespace mx {

// Sums of dy's columns over each expert's rows, 64 columns (from column `from` on) a workgroup.  16384 x 2048 bf16 among 8 experts 15.5 us (67 MB,
// 10 at memory's pace), 12 where the last-level cache still holds dy.
constexpr int kSumThreads = 1024;
template <class T>
__global__ __launch_bounds__(kSumThreads) void expert_sums_kernel(const T* __restrict__ dy, int64_t lddy, const int32_t* __restrict__ offsets, int64_t rows, int N, int from,
                                                                  float* __restrict__ db) {
    typedef ColumnSums<T, kSumThreads> Sums;
    __shared__ float shared[Sums::kFloats];
    int first, n;
    expert_rows(offsets, blockIdx.y, rows, first, n);
    Sums::run(dy, lddy, first, (int64_t)first + n, N, from + blockIdx.x * Sums::kColumns, db + (int64_t)blockIdx.y * N, shared);
}

static size_t dx_bytes(int64_t M, int experts) { return experts > kExpertsOfLanes ? table_bytes(M, experts) : 0; }
static bool grad_sizes_ok(int64_t M, int64_t N, int64_t K, int64_t experts) {
    return sizes_ok(M, K) && N >= 1 && N <= kMaxK && M < (1ll << 40) && experts_ok((int)experts);
}
static bool grad_countable(int64_t M, int64_t N, int experts) {
    return M < 1ll << 31 && experts <= SPARQ_MX_EXPERTS_MOST && experts * N < 1ll << 31;
}
static ExpertGradParams grad_params(const void* dy, int64_t lddy, const void* codes, const void* scales, int bits, int64_t ldo, int64_t J, int64_t R, int K,
                                    const int32_t* offsets, int64_t rows) {
    ExpertGradParams p = {};
    p.dy = dy;
    p.codes = static_cast<const uint8_t*>(codes);
    p.scales = static_cast<const uint8_t*>(scales);
    p.lddy = lddy;
    p.code_pitch = code_pitch(K, bits);
    p.scale_pitch = scale_pitch(K);
    p.ldo = ldo;
    p.J = J;
    p.R = R;
    p.K = K;
    p.K128 = (int)round_up(K, kCodeUnit);
    p.offsets = offsets;
    p.rows = rows;
    return p;
}
// Whether steps can be read without checks: the loads' offsets are 32 bits
static bool reads_fit(int64_t lddy, int64_t pitch) { return lddy < 1 << 21 && pitch < 1 << 24; }

}  // namespace mx
}  // namespace sparq

using namespace sparq;
using namespace sparq::mx;

extern "C" size_t sparq_mx_experts_dx_workspace_bytes(int64_t M, int32_t N, int32_t K, int32_t experts) {
    return grad_sizes_ok(M, N, K, experts) && M > 0 ? dx_bytes(M, experts) : 0;
}
extern "C" size_t sparq_mx_experts_dw_workspace_bytes(int64_t M, int32_t N, int32_t K, int32_t experts) {
    (void)M, (void)N, (void)K, (void)experts;
    return 0;
}

extern "C" sparq_status sparq_mx_experts_dx(const void* dy, int32_t dy_type, int64_t lddy, const int32_t* offsets, int32_t experts, const void* w_codes,
                                            const void* w_scales, void* dx, int32_t dx_type, int64_t lddx, int64_t M, int32_t N, int32_t K, void* workspace,
                                            size_t workspace_bytes, void* stream) {
    if (!grad_sizes_ok(M, N, K, experts) || !type_valid(dy_type) || (dx_type != dy_type && dx_type != SPARQ_MX_F32)) return SPARQ_EINVAL;
    if (!offsets || !aligned(offsets, 4)) return SPARQ_EINVAL;
    if (M == 0) return SPARQ_OK;
    if (!coded_ok(w_codes, w_scales) || !tensor_ok(dy, dy_type, lddy, N) || !tensor_ok(dx, dx_type, lddx, K)) return SPARQ_EINVAL;
    if (!extent_ok(M, lddy) || !extent_ok(M, lddx) || !extent_ok(M, K)) return SPARQ_EINVAL;
    const size_t bytes = dx_bytes(M, experts);
    if (bytes && (!workspace || !aligned(workspace, 256))) return SPARQ_EINVAL;
    if (workspace_bytes < bytes) return SPARQ_EWORKSPACE;
    const int t = dx_tile(dy_type, M, K, experts);
    const int64_t tiles_j = most_tiles(M, experts, t), tiles_k = (K + t - 1) / t, rest_k = (K + 63) / 64;
    if (!grad_countable(M, N, experts) || tiles_j * tiles_k * kGradThreads >= 1ll << 32) return SPARQ_EUNSUPPORTED;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (bytes) {
        const sparq_status tiled = launch_tiles(offsets, experts, M, t, workspace, s);
        if (tiled != SPARQ_OK) return tiled;
    }
    ExpertGradParams p = grad_params(dy, lddy, w_codes, w_scales, 4, lddx, M, N, K, offsets, M);
    p.table = bytes ? static_cast<const ExpertTile*>(workspace) : nullptr;
    p.experts = experts;
    p.s_whole = reads_fit(lddy, p.code_pitch) ? N / kGradStep : 0;
    p.steps_per_part = (N + kGradStep - 1) / kGradStep;
    const auto launch = [&](int tile, int64_t rows, int64_t columns) {
        p.tiles_k = (int)columns;
        return (dy_type == SPARQ_MX_F32 ? launch_experts_dx_f32 : dy_type == SPARQ_MX_F16 ? launch_experts_dx_f16 : launch_experts_dx_bf16)(
            p, dim3((unsigned)(rows * columns)), tile, dx, dx_type == SPARQ_MX_F32, s);
    };
    // Tiles of 256 x 256, one a CU at a time: where the experts' last ones, which are about half empty, would make a round more, what is left behind whole tiles goes in tiles
    // of 64, in a launch of its own (us, one launch -> two: 16384 x 2048 x 2048 to 8 experts, uneven, 149 -> 138, 16384 x 4096 x 1024 to 4 174 -> 130; the second takes 22 and 45, a step of
    // its 32 and 64 after the other).
    const int64_t half = (experts + 1) / 2, whole = M / 256 > half ? (M / 256 - half) * tiles_k : 0;
    if (t != 256 || bytes || rest_k * experts * 4 * kGradThreads >= 1ll << 32 || ((M / 256 + half) * tiles_k + 255) / 256 <= (whole + 255) / 256)
        return launch(t, tiles_j, tiles_k);
    p.whole = 256;
    const sparq_status done = launch(256, M / 256 > 0 ? M / 256 : 1, tiles_k);
    if (done != SPARQ_OK) return done;
    p.whole = -256;
    return launch(64, experts * 4ll, rest_k);
}

extern "C" sparq_status sparq_mx_experts_dw(const void* dy, int32_t dy_type, int64_t lddy, const int32_t* offsets, int32_t experts, const void* x_codes,
                                            const void* x_scales, void* dw, int32_t dw_type, int64_t lddw, float* db, int64_t M, int32_t N, int32_t K,
                                            void* workspace, size_t workspace_bytes, void* stream) {
    (void)workspace, (void)workspace_bytes;
    if (!grad_sizes_ok(M, N, K, experts) || !type_valid(dy_type) || (dw_type != dy_type && dw_type != SPARQ_MX_F32)) return SPARQ_EINVAL;
    if (!offsets || !aligned(offsets, 4)) return SPARQ_EINVAL;
    if (!tensor_ok(dw, dw_type, lddw, K) || !extent_ok((int64_t)experts * N, lddw) || !aligned(db, 4)) return SPARQ_EINVAL;
    if (M > 0 && (!coded_ok(x_codes, x_scales) || !tensor_ok(dy, dy_type, lddy, N) || !extent_ok(M, lddy) || !extent_ok(M, K))) return SPARQ_EINVAL;
    const int t = dw_tile(dy_type, M, N, K, experts);
    const int64_t tiles_j = (N + t - 1) / t, tiles_k = (K + t - 1) / t;
    // The column sums: by workgroups of the product's launch, which saves a launch, unless dy is so large that these would come last (as in
    // sparq_mx_grad.hip), or a workgroup of the tiles takes a CU for itself.
    constexpr int kColumns = ColumnSums<float, kGradThreads>::kColumns;
    const bool beside = db && M * N <= 1 << (t == 64 ? 22 : 21) && (dy_type == SPARQ_MX_BF16 || t == 64);
    const int64_t workgroups = tiles_j * tiles_k + (beside ? (N + kColumns - 1) / kColumns : 0);
    if (!grad_countable(M, N, experts) || workgroups * kGradThreads >= 1ll << 32) return SPARQ_EUNSUPPORTED;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    ExpertGradParams p = grad_params(dy, M > 0 ? lddy : 0, x_codes, x_scales, 8, lddw, N, 0, K, offsets, M);
    p.tiles_j = (int)tiles_j;
    p.tiles_k = (int)tiles_k;
    // A run that the last column cuts reads on into the next rows: the last rows, which it would leave, are not read in runs; none are if rows' distances do not
    // fit the loads' 32-bit offsets.
    p.margin = M == 0 ? 0 : reads_fit(lddy, p.code_pitch) ? (int)((round_up(N, 8) - N + lddy - 1) / lddy) : (int)M;
    p.experts = experts;
    p.column_sums = beside ? db : nullptr;
    const dim3 grid((unsigned)workgroups, (unsigned)experts);
    const sparq_status done = (dy_type == SPARQ_MX_F32 ? launch_experts_dw_f32 : dy_type == SPARQ_MX_F16 ? launch_experts_dw_f16 : launch_experts_dw_bf16)(
        p, grid, t, dw, dw_type == SPARQ_MX_F32, s);
    if (done != SPARQ_OK || !db || beside) return done;
    return in_launches((N + 63ll) / 64, kSumThreads, [&](int64_t first, int64_t n) {
        with_type(dy_type, [&](auto y) {
            typedef decltype(y) T;
            expert_sums_kernel<T><<<dim3((unsigned)n, (unsigned)experts), kSumThreads, 0, s>>>(static_cast<const T*>(dy), p.lddy, offsets, M, N, (int)(64 * first), db);
        });
        return launch_status();
    });
}
