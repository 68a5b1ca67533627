// The product's backward pass: dx over the 4-bit weights, dw over the 8-bit checkpoint (include/sparq_mx.h).
#include "sparq_mx_common.h"

namespace sparq {
namespace mx {

constexpr int kThreads = 256;

struct GradParams {
    const void* dy;
    const uint8_t *codes, *scales;
    int64_t lddy, code_pitch, scale_pitch, ldo;
    int64_t J, R;                        // results [J][K], sums of R products
    int32_t K;
};

// The bf16 parts of a value: their sum is the value (8 significand bits a part; 11 of fp16, 24 of fp32).
template <class T> constexpr int kParts = sizeof(T) == 4 ? 3 : 2;
template <> constexpr int kParts<__bf16> = 1;
template <int P>
__device__ __forceinline__ void split(float v, __bf16 (&part)[P]) {
    part[0] = (__bf16)v;
#pragma unroll
    for (int i = 1; i < P; ++i) {
        v -= (float)part[i - 1];
        part[i] = (__bf16)v;
    }
    if (P > 1 && !(__builtin_fabsf((float)part[0]) < __builtin_inff())) {    // NaN, infinity: nothing to add
#pragma unroll
        for (int i = 1; i < P; ++i) part[i] = (__bf16)0.0f;
    }
}

// out[j][k] = sum_r dy(j, r) * V[r][k].  DW: j = n, r = m, V = the 8-bit checkpoint; else j = m, r = n, V = the 4-bit weights.
// A wavefront makes 32 x 32 results; decoded values are bf16 exactly.
template <class T, class O, bool DW>
__global__ __launch_bounds__(kThreads) void grad_kernel(O* __restrict__ out, const GradParams p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 31, g = lane >> 5;
    const int k0 = (blockIdx.x * 2 + (wave & 1)) * 32, k = k0 + c < p.K ? k0 + c : p.K - 1;
    const int64_t j = ((int64_t)blockIdx.y * 2 + (wave >> 1)) * 32 + c, ja = j < p.J ? j : p.J - 1;
    const T* dy = static_cast<const T*>(p.dy);
    v16f acc = {};
    for (int64_t r0 = 0; r0 < p.R; r0 += 16) {
        v8bf V, D[kParts<T>];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const int64_t r = r0 + 8 * g + t;
            float v = 0.0f, d = 0.0f;
            if (r < p.R) {
                const uint32_t byte = p.scales[r * p.scale_pitch + (k >> 5)];
                if constexpr (DW) v = byte == 255 ? scale_value(byte) : __builtin_amdgcn_ldexpf((float)(int8_t)p.codes[r * p.code_pitch + k], (int)byte - 133);
                else {
                    const uint32_t q = p.codes[r * p.code_pitch + (k >> 1)] >> (4 * (k & 1));
                    v = byte == 255 ? scale_value(byte) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale_value(byte), 0)[0];
                }
                d = (float)(DW ? dy[r * p.lddy + ja] : dy[ja * p.lddy + r]);
            }
            V[t] = (__bf16)v;
            __bf16 part[kParts<T>];
            split(d, part);
#pragma unroll
            for (int i = 0; i < kParts<T>; ++i) D[i][t] = part[i];
        }
#pragma unroll
        for (int i = 0; i < kParts<T>; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(V, D[i], acc, 0, 0, 0);
    }
    if (j >= p.J) return;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int kk = k0 + 8 * (i >> 2) + 4 * g + (i & 3);
        if (kk < p.K) out[j * p.ldo + kk] = (O)acc[i];
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void column_sum_kernel(const T* __restrict__ dy, int64_t ld, int64_t rows, int n, float* __restrict__ sum) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= n) return;
    float s = 0.0f;
    for (int64_t r = 0; r < rows; ++r) s += (float)dy[r * ld + c];
    sum[c] = s;
}

template <bool DW>
static sparq_status launch_grad(const GradParams& p, int dy_type, void* out, int out_type, hipStream_t stream) {
    const dim3 grid((p.K + 63) / 64, (unsigned)((p.J + 63) / 64));
    with_type(dy_type, [&](auto t) {
        with_type(out_type, [&](auto o) {
            typedef decltype(t) T;
            typedef decltype(o) O;
            grad_kernel<T, O, DW><<<grid, kThreads, 0, stream>>>(static_cast<O*>(out), p);
        });
    });
    return launch_status();
}

static bool grad_sizes_ok(int64_t M, int64_t N, int64_t K) { return sizes_ok(M, K) && N >= 1 && N <= kMaxK; }

}  // namespace mx
}  // namespace sparq

using namespace sparq;
using namespace sparq::mx;

extern "C" size_t sparq_mx_linear_dx_workspace_bytes(int64_t, int32_t, int32_t) { return 0; }
extern "C" size_t sparq_mx_linear_dw_workspace_bytes(int64_t, int32_t, int32_t) { return 0; }

extern "C" sparq_status sparq_mx_linear_dx(const void* dy, int32_t dy_type, int64_t lddy, const void* w_codes, const void* w_scales,
                                           void* dx, int32_t dx_type, int64_t lddx, int64_t M, int32_t N, int32_t K,
                                           void* workspace, size_t workspace_bytes, void* stream) {
    if (!grad_sizes_ok(M, N, K) || !type_valid(dy_type) || !type_valid(dx_type)) return SPARQ_EINVAL;
    if (M == 0) return SPARQ_OK;
    if (!coded_ok(w_codes, w_scales) || !tensor_ok(dy, dy_type, lddy, N) || !tensor_ok(dx, dx_type, lddx, K)) return SPARQ_EINVAL;
    if (!extent_ok(M, lddy) || !extent_ok(M, lddx)) return SPARQ_EINVAL;
    if (M > 65535 * 64ll) return SPARQ_EUNSUPPORTED;
    const GradParams p = {dy, static_cast<const uint8_t*>(w_codes), static_cast<const uint8_t*>(w_scales), lddy, code_pitch(K, 4),
                          scale_pitch(K), lddx, M, N, K};
    return launch_grad<false>(p, dy_type, dx, dx_type, static_cast<hipStream_t>(stream));
}

extern "C" sparq_status sparq_mx_linear_dw(const void* dy, int32_t dy_type, int64_t lddy, const void* x_codes, const void* x_scales,
                                           void* dw, int32_t dw_type, int64_t lddw, float* db, int64_t M, int32_t N, int32_t K,
                                           void* workspace, size_t workspace_bytes, void* stream) {
    if (!grad_sizes_ok(M, N, K) || !type_valid(dy_type) || !type_valid(dw_type)) return SPARQ_EINVAL;
    if (!tensor_ok(dw, dw_type, lddw, K) || !extent_ok(N, lddw) || !aligned(db, 4)) return SPARQ_EINVAL;
    if (M > 0 && (!coded_ok(x_codes, x_scales) || !tensor_ok(dy, dy_type, lddy, N) || !extent_ok(M, lddy) || !extent_ok(M, K)))
        return SPARQ_EINVAL;
    if (N > 65535 * 64) return SPARQ_EUNSUPPORTED;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (db)
        with_type(dy_type, [&](auto t) {
            typedef decltype(t) T;
            column_sum_kernel<T><<<(N + kThreads - 1) / kThreads, kThreads, 0, s>>>(static_cast<const T*>(dy), lddy, M, N, db);
        });
    const GradParams p = {dy, static_cast<const uint8_t*>(x_codes), static_cast<const uint8_t*>(x_scales), lddy, code_pitch(K, 8),
                          scale_pitch(K), lddw, N, M, K};
    return launch_grad<true>(p, dy_type, dw, dw_type, s);
}
