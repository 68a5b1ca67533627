// Dropout from a counter-based generator, and the residual it is added to (include/sparq_mx_experts.h).
#include "sparq_mx_experts.h"

namespace sparq {
namespace mx {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

struct DropoutParams {
    int64_t ldx, ldr, ldy;
    uint64_t seed, offset, first_group;  // first_group: of the launch's first row
    const uint64_t* step;
    uint32_t limit;                      // bits below this are dropped
    float scale;
    int32_t K;
    uint32_t groups, items, chunks;      // groups of eight in a row; wavefronts' worth of work: rows x chunks of 512 values
    FastDiv div_chunks;
};

// Philox 4x32, ten rounds.
__device__ __forceinline__ v4u random_words(uint64_t counter_low, uint64_t counter_high, uint64_t key) {
    uint32_t c0 = (uint32_t)counter_low, c1 = (uint32_t)(counter_low >> 32), c2 = (uint32_t)counter_high, c3 = (uint32_t)(counter_high >> 32);
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return v4u{c0, c1, c2, c3};
}

// A wavefront takes 512 values of a row, a lane eight: one call of the generator, twenty products of 32 x 32 bits, which is half of what the vector units have time for
// while the values pass.  (32 bits an element would take two calls and all of it.)  Bound by memory: 16384 x 4096 bf16 with a residual 62 us (6.5 TB/s), without
// 43 (6.2); fp32 134 and 94 (6.0, 5.7).
template <class T, bool RESIDUAL, int STREAMING>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const T* __restrict__ x, const T* __restrict__ residual, T* __restrict__ y, const DropoutParams p) {
    const int lane = threadIdx.x & 63;
    const uint32_t item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= p.items) return;
    const uint32_t row = fastdiv(item, p.div_chunks);
    const int col = (int)(item - row * p.chunks) * kScaleUnit + 8 * lane, n = p.K - col;
    if (n <= 0) return;
    float v[8], r[8];
    load_upto8<STREAMING == kAll>(x + row * p.ldx + col, n, v);
    if constexpr (RESIDUAL) load_upto8<STREAMING == kAll>(residual + row * p.ldr + col, n, r);
    const uint64_t offset = p.offset + (p.step ? *p.step : 0);
    const v4u words = random_words(p.first_group + (uint64_t)row * p.groups + (uint32_t)(col >> 3), offset, p.seed);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = words[i >> 1] >> (16 * (i & 1)) & 0xFFFFu;
        const float kept = bits >= p.limit ? v[i] * p.scale : 0.0f;
        v[i] = RESIDUAL ? r[i] + kept : kept;
    }
    store_upto8<STREAMING != kKept>(y + row * p.ldy + col, n, v);
}

}  // namespace mx
}  // namespace sparq

using namespace sparq;
using namespace sparq::mx;

extern "C" sparq_status sparq_mx_dropout(const void* x, int64_t ldx, double p, uint64_t seed, uint64_t offset, const uint64_t* step, const void* residual,
                                         int64_t ldr, void* y, int64_t ldy, int32_t type, int64_t rows, int32_t K, void* stream) {
    if (!sizes_ok(rows, K) || !type_valid(type) || !(p >= 0.0 && p <= 1.0)) return SPARQ_EINVAL;
    if (rows == 0) return SPARQ_OK;
    if (!tensor_ok(x, type, ldx, K) || !tensor_ok(y, type, ldy, K) || (residual && !tensor_ok(residual, type, ldr, K)) || !aligned(step, 8)) return SPARQ_EINVAL;
    if (!extent_ok(rows, ldx) || !extent_ok(rows, ldy) || (residual && !extent_ok(rows, ldr)) || !extent_ok(rows, K)) return SPARQ_EINVAL;
    const int64_t chunks = (K + kScaleUnit - 1) / kScaleUnit, items = rows * chunks;
    if (rows >= (1ll << 31) || items >= (1ll << 31)) return SPARQ_EUNSUPPORTED;
    const uint32_t limit = (uint32_t)__builtin_rint(p * 65536.0);
    const DropoutParams all = {ldx, ldr, ldy, seed, offset, 0, step, limit, limit < 65536 ? (float)(65536.0 / (65536 - (int)limit)) : 0.0f, K,
                               (uint32_t)((K + 7) / 8), (uint32_t)items, (uint32_t)chunks, make_fastdiv((uint32_t)chunks)};
    sparq_status s = SPARQ_OK;
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const int64_t result = rows * K * (int64_t)sizeof(T);
        with_streaming<T>((residual ? 3 : 2) * result, result, [&](auto streaming) {
            constexpr int S = decltype(streaming)::value;
            const auto kernel = residual ? dropout_kernel<T, true, S> : dropout_kernel<T, false, S>;
            s = in_launches(rows, 64 * chunks, [&](int64_t first, int64_t n) {
                DropoutParams q = all;
                q.first_group = (uint64_t)first * all.groups;
                q.items = (uint32_t)(n * chunks);
                kernel<<<(q.items + kWaves - 1) / kWaves, kThreads, 0, static_cast<hipStream_t>(stream)>>>(
                    static_cast<const T*>(x) + first * ldx, residual ? static_cast<const T*>(residual) + first * ldr : nullptr, static_cast<T*>(y) + first * ldy, q);
                return launch_status();
            });
        });
    });
    return s;
}
