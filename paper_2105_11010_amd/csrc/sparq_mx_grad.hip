// The product's backward pass: entry points, the choice of tiles, and the sums that join a divided reduction.
#include "sparq_mx_grad.h"

namespace sparq {
namespace mx {

// Sums of dy's columns from `first` on, a grid row a slab of its rows, for gradients as large as to keep memory busy on their own.
constexpr int kSumThreads = 1024;
template <class T>
__global__ __launch_bounds__(kSumThreads) void column_sum_kernel(const GradParams p, int first) {
    typedef ColumnSums<T, kSumThreads> Sums;
    __shared__ float shared[Sums::kFloats];
    const int64_t begin = blockIdx.y * p.slab, end = begin + p.slab < p.R ? begin + p.slab : p.R;
    Sums::run(static_cast<const T*>(p.dy), p.lddy, begin, end, (int)p.J, first + blockIdx.x * Sums::kColumns, p.column_sums + blockIdx.y * p.J, shared);
}

// ---- plan ----------------------------------------------------------------------------
struct GradPlan {
    int tile;                // 256 (bf16), 128 or 64: results a workgroup makes along either side
    int parts;               // of the reduction
    int slabs;               // of rows for the column sums
    size_t partial_bytes, bytes;
};
static GradPlan grad_plan(int dy_type, int64_t J, int64_t R, int K, bool dw) {
    GradPlan p = {};
    const auto tiles = [&](int t) { return ((J + t - 1) / t) * ((K + t - 1) / t); };
    // 256 x 256 results, one such tile a CU at a time, or 128 x 128, two a CU: by the rounds that 256 CUs make of them, of which the former's last half
    // as long again (us, 256 -> 128: dx 4096^3 110 -> 144, 3000^3 68 -> 87, 2048^3 42 -> 22; dw 134 -> 168, 85 -> 102, 57 -> 32, of 4096 x 2048 x 4096
    // 107 -> 84); dw of a few rows is all results, which two workgroups a CU write better than one (64 x 8192 x 8192 63 -> 47, 256 x 4096 x 4096 24 -> 21).
    // 64 x 64 where those leave CUs without (128 -> 64: dx 2048^3 24 -> 34, dw 8192 x 1024 x 1024 35 -> 57, 1024 x 4096 x 1024 18 -> 22).
    const bool bf16 = dy_type == SPARQ_MX_BF16;
    const int64_t least = (bf16 ? 16 : dy_type == SPARQ_MX_F16 ? 8 : 6) >> (J * K <= 1 << 17 ? 1 : 0);       // steps of a part, by what one takes
    const int64_t steps = (R + kGradStep - 1) / kGradStep, most = steps / least > 1 ? steps / least : 1;
    p.tile = bf16 && !(dw && steps <= 4) && 3 * ((tiles(256) + 255) / 256) <= 2 * ((tiles(128) + 511) / 512) ? 256 : tiles(128) * most >= 192 ? 128 : 64;
    // Few tiles of a long reduction are divided, into as many parts of at least `least` steps as there is room for (us, of 16 steps -> of these: dw 1648
    // x 217 x 55 fp16 20.7 -> 12.3, 1757 x 1234 x 114 fp32 31 -> 17, 1664 x 17 x 39 bf16 13.5 -> 10.4; dx 24 x 3008 x 49 fp16 18.9 -> 13.0; bf16 in parts of
    // eight where there are more results: 700 x 1100 x 900 10 -> 14); shorter ones are over before the parts would be joined, and tiles that fill
    // most CUs gain from two parts only if those are long (whole -> two parts: dw 8192 x 3000 x 1000 114 -> 90, 8192 x 2048 x 2048 120 -> 106; dx
    // 2048^3 24 -> 27).
    const int64_t n = tiles(p.tile), places = (p.tile == 128 ? (bf16 ? 512 : 256) : 1024) / n, parts = places < most ? places : most;
    const bool divided = p.tile != 256 && (n < 192 || (n <= 256 && steps >= 64));
    p.parts = !divided || parts < 1 ? 1 : (int)(parts > 64 ? 64 : parts);
    const int64_t columns = (J + 63) / 64, slabs = R / 512 < 1024 / columns ? R / 512 : 1024 / columns;
    p.slabs = !dw ? 0 : slabs < 1 ? 1 : (int)slabs;
    p.partial_bytes = p.parts > 1 ? (size_t)round_up(p.parts * J * K * 4, 256) : 0;
    p.bytes = p.partial_bytes + (p.slabs > 1 ? (size_t)round_up((int64_t)p.slabs * J * 4, 256) : 0);
    return p;
}
// The workspace does not depend on dy's type: the largest.
static size_t grad_bytes(int64_t J, int64_t R, int K, bool dw) {
    size_t most = 0;
    for (const int type : {SPARQ_MX_F32, SPARQ_MX_F16, SPARQ_MX_BF16}) {
        const size_t bytes = grad_plan(type, J, R, K, dw).bytes;
        most = bytes > most ? bytes : most;
    }
    return most;
}
// Steps that are read without checks, in runs of eight: none if rows' distances do not fit the loads' 32-bit offsets.  A run that dw's last
// column cuts reads on into the next rows (one, unless rows are shorter than a run): the last rows, which it would leave, are not among them.
static int64_t whole_steps(int64_t lddy, int64_t J, int64_t R, int64_t pitch, bool dw) {
    if (R == 0 || lddy >= 1 << 21 || pitch >= 1 << 24 || R >= 1ll << 36) return 0;       // (of no rows lddy may be anything)
    const int64_t over = dw ? round_up(J, 8) - J : 0, rows = R - (over + lddy - 1) / lddy;
    return rows > 0 ? rows / kGradStep : 0;
}

static sparq_status grad(const void* dy, int dy_type, int64_t lddy, const void* codes, const void* scales, int bits, void* out, int out_type,
                         int64_t ldo, float* column_sums, int64_t J, int64_t R, int K, const GradPlan& plan, void* workspace, hipStream_t stream) {
    const int t = plan.tile;
    const int64_t tiles_j = (J + t - 1) / t, tiles_k = (K + t - 1) / t;
    // (dw's rows and columns are at most 2^28: more tiles than one launch takes would be results of half a terabyte)
    constexpr int kColumns = ColumnSums<float, kGradThreads>::kColumns;
    if (bits == 8 && (tiles_j * tiles_k + (column_sums ? plan.slabs : 0) * ((J + kColumns - 1) / kColumns)) * kGradThreads >= 1ll << 32) return SPARQ_EUNSUPPORTED;
    GradParams p = {};
    p.dy = dy;
    p.codes = static_cast<const uint8_t*>(codes);
    p.scales = static_cast<const uint8_t*>(scales);
    p.lddy = lddy;
    p.code_pitch = code_pitch(K, bits);
    p.scale_pitch = scale_pitch(K);
    p.J = J;
    p.R = R;
    p.K = K;
    p.K128 = (int)round_up(K, kCodeUnit);
    p.column_sums = column_sums;
    p.slab = plan.slabs > 1 ? (R + plan.slabs - 1) / plan.slabs : R;
    p.slabs = column_sums ? plan.slabs : 0;
    // The column sums: by workgroups of the product's launch, which saves a launch, unless dy is so large that these would come last and
    // last longer than it (us with either, in the launch -> in one before: 515 x 771 x 577 8.4 -> 13.4, 2048^3 36.9 -> 40.8, 4096 x 512 x 512
    // 16.8 -> 20.3; 8192 x 1024 x 1024 45.6 -> 42.5, 4096^3 150 -> 141, 8192 x 4096 x 4096 283 -> 272).
    if (column_sums && J * R > 1 << 22) {
        const sparq_status s = in_launches((J + 63) / 64, kSumThreads, [&](int64_t first, int64_t n) {
            with_type(dy_type, [&](auto t) { column_sum_kernel<decltype(t)><<<dim3((unsigned)n, p.slabs), kSumThreads, 0, stream>>>(p, (int)(64 * first)); });
            return launch_status();
        });
        p.slabs = 0;
        if (s != SPARQ_OK) return s;
    }
    p.s_whole = whole_steps(lddy, J, R, p.code_pitch, bits == 8);
    const int64_t steps = (R + kGradStep - 1) / kGradStep;
    p.tiles_k = (int)tiles_k;
    p.steps_per_part = (int)((steps + plan.parts - 1) / plan.parts);
    const bool parted = plan.parts > 1;
    p.ldo = parted ? K : ldo;
    p.part_stride = parted ? J * K : 0;
    void* const to = parted ? workspace : out;
    const int to_type = parted ? SPARQ_MX_F32 : out_type;
    sparq_status s;
    if (bits == 8) {
        p.tiles_j = (int)tiles_j;
        s = launch_grad(p, plan.parts, t, dy_type, true, to, to_type, stream);
    } else {
        // (more than one launch: no parts)
        s = in_launches(tiles_j, tiles_k * kGradThreads, [&](int64_t first, int64_t n) {
            GradParams q = p;                                // of the rows from here on
            const int64_t row = first * t;
            q.dy = static_cast<const char*>(dy) + row * lddy * (int64_t)type_bytes(dy_type);
            q.J -= row;
            q.tiles_j = (int)n;
            return launch_grad(q, plan.parts, t, dy_type, false, static_cast<char*>(to) + row * p.ldo * (int64_t)type_bytes(to_type), to_type, stream);
        });
    }
    if (s != SPARQ_OK || !parted) return s;
    return launch_join(static_cast<const float*>(workspace), nullptr, out, out_type, J, K, ldo, plan.parts, stream);
}

static bool grad_sizes_ok(int64_t M, int64_t N, int64_t K) { return sizes_ok(M, K) && N >= 1 && N <= kMaxK && M < (1ll << 40); }

}  // namespace mx
}  // namespace sparq

using namespace sparq;
using namespace sparq::mx;

extern "C" size_t sparq_mx_linear_dx_workspace_bytes(int64_t M, int32_t N, int32_t K) {
    return grad_sizes_ok(M, N, K) && extent_ok(M, K) && M > 0 ? grad_bytes(M, N, K, false) : 0;
}
extern "C" size_t sparq_mx_linear_dw_workspace_bytes(int64_t M, int32_t N, int32_t K) {
    return grad_sizes_ok(M, N, K) ? grad_bytes(N, M, K, true) : 0;
}

extern "C" sparq_status sparq_mx_linear_dx(const void* dy, int32_t dy_type, int64_t lddy, const void* w_codes, const void* w_scales,
                                           void* dx, int32_t dx_type, int64_t lddx, int64_t M, int32_t N, int32_t K,
                                           void* workspace, size_t workspace_bytes, void* stream) {
    if (!grad_sizes_ok(M, N, K) || !type_valid(dy_type) || !type_valid(dx_type)) return SPARQ_EINVAL;
    if (M == 0) return SPARQ_OK;
    if (!coded_ok(w_codes, w_scales) || !tensor_ok(dy, dy_type, lddy, N) || !tensor_ok(dx, dx_type, lddx, K)) return SPARQ_EINVAL;
    if (!extent_ok(M, lddy) || !extent_ok(M, lddx) || !extent_ok(M, K)) return SPARQ_EINVAL;
    const GradPlan plan = grad_plan(dy_type, M, N, K, false);
    if (plan.bytes && (!workspace || !aligned(workspace, 256))) return SPARQ_EINVAL;
    if (workspace_bytes < plan.bytes) return SPARQ_EWORKSPACE;
    return grad(dy, dy_type, lddy, w_codes, w_scales, 4, dx, dx_type, lddx, nullptr, M, N, K, plan, workspace, static_cast<hipStream_t>(stream));
}

extern "C" sparq_status sparq_mx_linear_dw(const void* dy, int32_t dy_type, int64_t lddy, const void* x_codes, const void* x_scales,
                                           void* dw, int32_t dw_type, int64_t lddw, float* db, int64_t M, int32_t N, int32_t K,
                                           void* workspace, size_t workspace_bytes, void* stream) {
    if (!grad_sizes_ok(M, N, K) || !type_valid(dy_type) || !type_valid(dw_type)) return SPARQ_EINVAL;
    if (!tensor_ok(dw, dw_type, lddw, K) || !extent_ok(N, lddw) || !aligned(db, 4)) return SPARQ_EINVAL;
    if (M > 0 && (!coded_ok(x_codes, x_scales) || !tensor_ok(dy, dy_type, lddy, N) || !extent_ok(M, lddy) || !extent_ok(M, K)))
        return SPARQ_EINVAL;
    const GradPlan plan = grad_plan(dy_type, N, M, K, true);
    if (plan.bytes && (!workspace || !aligned(workspace, 256))) return SPARQ_EINVAL;
    if (workspace_bytes < plan.bytes) return SPARQ_EWORKSPACE;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool slabs = db && plan.slabs > 1;
    float* const sums = slabs ? reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.partial_bytes) : db;
    const sparq_status done = grad(dy, dy_type, lddy, x_codes, x_scales, 8, dw, dw_type, lddw, sums, N, M, K, plan, workspace, s);
    return done != SPARQ_OK || !slabs ? done : launch_join_columns(sums, db, nullptr, N, N, plan.slabs, s);
}
