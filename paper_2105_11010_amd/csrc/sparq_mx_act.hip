// Gated activations with 8-bit checkpoints of their inputs, and their backward pass from those (include/sparq_mx.h).
#include <type_traits>

#include "sparq_mx_function.h"

namespace sparq {
namespace mx {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

struct ActParams {
    int64_t ldg, ldu, ldy, code_pitch, scale_pitch;
    int32_t K, K128;
    uint32_t items, chunks;              // wavefronts' worth of work: rows x chunks of 512 values
    FastDiv div_chunks;
};

// A wavefront takes 512 values of a row, a lane eight, as the quantiser does.  8192 x 8192 bf16, gated, with both checkpoints: silu 83 us
// (6.5 TB/s), bound by memory, as is its gradient (83); gelu 93-95 and 87-89, bound by its arithmetic; fp32 silu 163 and 170, gelu 164 and 179.
template <class T, int F, bool UP, bool KEEP, int STREAMING>
__global__ __launch_bounds__(kThreads) void act_kernel(const T* __restrict__ gate, const T* __restrict__ up, T* __restrict__ y,
                                                       uint8_t* __restrict__ gate_codes, uint8_t* __restrict__ gate_scales,
                                                       uint8_t* __restrict__ up_codes, uint8_t* __restrict__ up_scales, const ActParams p) {
    const int lane = threadIdx.x & 63;
    const uint32_t item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= p.items) return;
    const uint32_t row = fastdiv(item, p.div_chunks);
    const int col = (int)(item - row * p.chunks) * kScaleUnit + 8 * lane, n = p.K - col;
    float g[8], u[8], o[8];
    load_upto8<STREAMING == kAll>(gate + row * p.ldg + col, n, g);
    if constexpr (UP) load_upto8<STREAMING == kAll>(up + row * p.ldu + col, n, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = function<F, sizeof(T) == 4>(g[i]) * (UP ? u[i] : 1.0f);
    if (n > 0) store_upto8<STREAMING != kKept>(y + row * p.ldy + col, n, o);
    if constexpr (KEEP) {
        const int64_t codes_at = row * p.code_pitch + col, scale_at = row * p.scale_pitch + (col >> 5);
        auto keep = [&](const float (&v)[8], uint8_t* codes, uint8_t* scales) __attribute__((always_inline)) {
            const uint32_t byte = scale8_of(block_top(v));
            const v2u w = codes8_of(v, byte);
            if (col < p.K128) *reinterpret_cast<v2u*>(codes + codes_at) = w;
            if ((lane & 3) == 0) scales[scale_at] = (uint8_t)byte;
        };
        if (gate_codes) keep(g, gate_codes, gate_scales);
        if constexpr (UP)
            if (up_codes) keep(u, up_codes, up_scales);
    }
}

template <class T, int F, bool UP, int STREAMING>
__global__ __launch_bounds__(kThreads) void act_grad_kernel(const T* __restrict__ dy, const uint8_t* __restrict__ gate_codes,
                                                            const uint8_t* __restrict__ gate_scales, const uint8_t* __restrict__ up_codes,
                                                            const uint8_t* __restrict__ up_scales, T* __restrict__ dgate,
                                                            T* __restrict__ dup, const ActParams p) {
    const int lane = threadIdx.x & 63;
    const uint32_t item = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= p.items) return;
    const uint32_t row = fastdiv(item, p.div_chunks);
    const int col = (int)(item - row * p.chunks) * kScaleUnit + 8 * lane, n = p.K - col;
    if (n <= 0) return;
    const int64_t codes_at = row * p.code_pitch + col, scale_at = row * p.scale_pitch + (col >> 5);
    float d[8], g[8], u[8], dg[8], du[8];
    load_upto8<STREAMING == kAll>(dy + row * p.ldy + col, n, d);
    values8_of(*reinterpret_cast<const v2u*>(gate_codes + codes_at), gate_scales[scale_at], g);
    if constexpr (UP) values8_of(*reinterpret_cast<const v2u*>(up_codes + codes_at), up_scales[scale_at], u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float value, slope;
        function_and_slope<F, sizeof(T) == 4>(g[i], value, slope);
        dg[i] = (UP ? d[i] * u[i] : d[i]) * slope;
        du[i] = d[i] * value;
    }
    store_upto8<STREAMING != kKept>(dgate + row * p.ldg + col, n, dg);
    if constexpr (UP) store_upto8<STREAMING != kKept>(dup + row * p.ldu + col, n, du);
}

static bool act_params(int64_t rows, int K, int64_t ldg, int64_t ldu, int64_t ldy, ActParams* p) {
    const int64_t chunks = (K + kScaleUnit - 1) / kScaleUnit, items = rows * chunks;
    if (rows >= (1ll << 31) || items >= (1ll << 31)) return false;
    *p = {ldg, ldu, ldy, code_pitch(K, 8), scale_pitch(K), K, (int)round_up(K, kCodeUnit), (uint32_t)items, (uint32_t)chunks,
          make_fastdiv((uint32_t)chunks)};
    return true;
}
// f(p, grid, first): launches for the rows from `first` on, p of as many of them as a launch takes
template <class F>
static sparq_status in_act_launches(int64_t rows, ActParams p, F&& f) {
    return in_launches(rows, 64ll * p.chunks, [&](int64_t first, int64_t n) {
        p.items = (uint32_t)(n * p.chunks);
        f(p, (p.items + kWaves - 1) / kWaves, first);
        return launch_status();
    });
}
static bool function_valid(int f) { return f == SPARQ_MX_SILU || f == SPARQ_MX_GELU; }

}  // namespace mx
}  // namespace sparq

using namespace sparq;
using namespace sparq::mx;

extern "C" sparq_status sparq_mx_act(int32_t function, const void* gate, int64_t ldg, const void* up, int64_t ldu, void* y, int64_t ldy,
                                     int32_t type, void* gate_codes, void* gate_scales, void* up_codes, void* up_scales, int64_t rows,
                                     int32_t K, void* stream) {
    if (!function_valid(function) || !sizes_ok(rows, K) || !type_valid(type)) return SPARQ_EINVAL;
    if (rows == 0) return SPARQ_OK;
    if (!tensor_ok(gate, type, ldg, K) || (up && !tensor_ok(up, type, ldu, K)) || !tensor_ok(y, type, ldy, K)) return SPARQ_EINVAL;
    if (!extent_ok(rows, ldg) || (up && !extent_ok(rows, ldu)) || !extent_ok(rows, ldy) || !extent_ok(rows, K)) return SPARQ_EINVAL;
    if (!coded_ok_or_none(gate_codes, gate_scales) || !coded_ok_or_none(up_codes, up_scales) || (up_codes && !up)) return SPARQ_EINVAL;
    ActParams p;
    if (!act_params(rows, K, ldg, ldu, ldy, &p)) return SPARQ_EUNSUPPORTED;
    sparq_status s = SPARQ_OK;
    const bool keep = gate_codes || up_codes;
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const auto launch = [&](auto kernel) {
            s = in_act_launches(rows, p, [&](const ActParams& q, uint32_t grid, int64_t first) {
                kernel<<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(
                    static_cast<const T*>(gate) + first * ldg, up ? static_cast<const T*>(up) + first * ldu : nullptr, static_cast<T*>(y) + first * ldy,
                    row_of(gate_codes, first, p.code_pitch), row_of(gate_scales, first, p.scale_pitch), row_of(up_codes, first, p.code_pitch),
                    row_of(up_scales, first, p.scale_pitch), q);
            });
        };
        const auto of = [&](auto f) {
            constexpr int F = decltype(f)::value;
            const int64_t result = rows * K * (int64_t)sizeof(T);
            with_streaming<T>((up ? 3 : 2) * result + rows * K * ((gate_codes ? 1 : 0) + (up_codes ? 1 : 0)), result, [&](auto streaming) {
                constexpr int S = decltype(streaming)::value;
                if (up) keep ? launch(act_kernel<T, F, true, true, S>) : launch(act_kernel<T, F, true, false, S>);
                else keep ? launch(act_kernel<T, F, false, true, S>) : launch(act_kernel<T, F, false, false, S>);
            });
        };
        if (function == SPARQ_MX_SILU) of(std::integral_constant<int, SPARQ_MX_SILU>{});
        else of(std::integral_constant<int, SPARQ_MX_GELU>{});
    });
    return s;
}

extern "C" sparq_status sparq_mx_act_grad(int32_t function, const void* dy, int64_t lddy, const void* gate_codes, const void* gate_scales,
                                          const void* up_codes, const void* up_scales, void* dgate, int64_t lddg, void* dup, int64_t lddu,
                                          int32_t type, int64_t rows, int32_t K, void* stream) {
    if (!function_valid(function) || !sizes_ok(rows, K) || !type_valid(type)) return SPARQ_EINVAL;
    if (rows == 0) return SPARQ_OK;
    const bool up = up_codes || up_scales || dup;
    if (!tensor_ok(dy, type, lddy, K) || !tensor_ok(dgate, type, lddg, K) || (up && !tensor_ok(dup, type, lddu, K))) return SPARQ_EINVAL;
    if (!extent_ok(rows, lddy) || !extent_ok(rows, lddg) || (up && !extent_ok(rows, lddu)) || !extent_ok(rows, K)) return SPARQ_EINVAL;
    if (!coded_ok(gate_codes, gate_scales) || (up && !coded_ok(up_codes, up_scales))) return SPARQ_EINVAL;
    ActParams p;
    if (!act_params(rows, K, lddg, lddu, lddy, &p)) return SPARQ_EUNSUPPORTED;
    sparq_status s = SPARQ_OK;
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const auto launch = [&](auto kernel) {
            s = in_act_launches(rows, p, [&](const ActParams& q, uint32_t grid, int64_t first) {
                kernel<<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(
                    static_cast<const T*>(dy) + first * lddy, row_of(gate_codes, first, p.code_pitch), row_of(gate_scales, first, p.scale_pitch),
                    row_of(up_codes, first, p.code_pitch), row_of(up_scales, first, p.scale_pitch), static_cast<T*>(dgate) + first * lddg,
                    up ? static_cast<T*>(dup) + first * lddu : nullptr, q);
            });
        };
        const auto of = [&](auto f) {
            constexpr int F = decltype(f)::value;
            const int64_t result = rows * K * (int64_t)sizeof(T);
            with_streaming<T>((up ? 3 : 2) * result + rows * K * (up ? 2 : 1), (up ? 2 : 1) * result, [&](auto streaming) {
                constexpr int S = decltype(streaming)::value;
                up ? launch(act_grad_kernel<T, F, true, S>) : launch(act_grad_kernel<T, F, false, S>);
            });
        };
        if (function == SPARQ_MX_SILU) of(std::integral_constant<int, SPARQ_MX_SILU>{});
        else of(std::integral_constant<int, SPARQ_MX_GELU>{});
    });
    return s;
}
