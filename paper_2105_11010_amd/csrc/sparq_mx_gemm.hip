// The product of 4-bit operands (include/sparq_mx.h).
#include "sparq_mx_common.h"

namespace sparq {
namespace mx {

constexpr int kThreads = 256;

struct GemmParams {
    const uint8_t *a, *as, *w, *ws;
    const float* bias;
    int64_t M, ldy, code_pitch, scale_pitch;
    int32_t N, steps;                    // steps of 64 values
};

// y[m][n] = sum_k W[n][k] A[m][k] on v_mfma_scale_f32_32x32x64: a lane feeds 32 values of one row, i.e. one block and its
// scale.  The weights are the instruction's first operand, so that a lane ends with four neighbouring n of one m.
// A wavefront makes 32 x 32 results from operands read where they are.
template <class T>
__global__ __launch_bounds__(kThreads) void gemm_kernel(T* __restrict__ y, const GemmParams p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, g = lane >> 5;
    const int64_t m = ((int64_t)blockIdx.y * 2 + (wave >> 1)) * 32 + r;
    const int n0 = (blockIdx.x * 2 + (wave & 1)) * 32;
    const int64_t ma = m < p.M ? m : p.M - 1;
    const int na = n0 + r < p.N ? n0 + r : p.N - 1;
    const uint8_t *a = p.a + ma * p.code_pitch + 16 * g, *as = p.as + ma * p.scale_pitch + g;
    const uint8_t *w = p.w + na * p.code_pitch + 16 * g, *ws = p.ws + na * p.scale_pitch + g;
    v16f acc = {};
    for (int s = 0; s < p.steps; ++s) {
        const v4i av = *reinterpret_cast<const v4i*>(a + 32 * (int64_t)s), wv = *reinterpret_cast<const v4i*>(w + 32 * (int64_t)s);
        const v8i A = {av[0], av[1], av[2], av[3], 0, 0, 0, 0}, W = {wv[0], wv[1], wv[2], wv[3], 0, 0, 0, 0};
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(W, A, acc, 4, 4, 0, ws[2 * s], 0, as[2 * s]);
    }
    if (m >= p.M) return;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int n = n0 + 8 * (i >> 2) + 4 * g + (i & 3);
        if (n < p.N) y[m * p.ldy + n] = (T)(acc[i] + (p.bias ? p.bias[n] : 0.0f));
    }
}

sparq_status launch_gemm(const GemmParams& p, void* y, int type, hipStream_t stream) {
    const dim3 grid((p.N + 63) / 64, (unsigned)((p.M + 63) / 64));
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        gemm_kernel<T><<<grid, kThreads, 0, stream>>>(static_cast<T*>(y), p);
    });
    return launch_status();
}

static bool gemm_sizes_ok(int64_t M, int64_t N, int64_t K) { return sizes_ok(M, K) && N >= 1 && N <= kMaxK; }

}  // namespace mx
}  // namespace sparq

using namespace sparq;
using namespace sparq::mx;

extern "C" size_t sparq_mx_gemm_workspace_bytes(int64_t, int32_t, int32_t) { return 0; }

extern "C" sparq_status sparq_mx_gemm(const void* a_codes, const void* a_scales, const void* w_codes, const void* w_scales,
                                      const float* bias, void* y, int32_t type, int64_t ldy, int64_t M, int32_t N, int32_t K,
                                      void* workspace, size_t workspace_bytes, void* stream) {
    if (!gemm_sizes_ok(M, N, K) || !type_valid(type)) return SPARQ_EINVAL;
    if (M == 0) return SPARQ_OK;
    if (!coded_ok(a_codes, a_scales) || !coded_ok(w_codes, w_scales) || !aligned(bias, 4)) return SPARQ_EINVAL;
    if (!tensor_ok(y, type, ldy, N) || !extent_ok(M, ldy) || !extent_ok(M, K)) return SPARQ_EINVAL;
    if (M > 65535 * 64ll) return SPARQ_EUNSUPPORTED;
    const GemmParams p = {static_cast<const uint8_t*>(a_codes), static_cast<const uint8_t*>(a_scales), static_cast<const uint8_t*>(w_codes),
                          static_cast<const uint8_t*>(w_scales), bias, M, ldy, code_pitch(K, 4), scale_pitch(K), N, (K + 63) / 64};
    return launch_gemm(p, y, type, static_cast<hipStream_t>(stream));
}

static size_t coded_bytes(int64_t M, int K) { return (size_t)(round_up(M * code_pitch(K, 4), 256) + round_up(M * scale_pitch(K), 256)); }

extern "C" size_t sparq_mx_linear_workspace_bytes(int64_t M, int32_t N, int32_t K) {
    return gemm_sizes_ok(M, N, K) && extent_ok(M, K) ? coded_bytes(M, K) : 0;
}

extern "C" sparq_status sparq_mx_linear(const void* x, int32_t x_type, int64_t ldx, const void* w_codes, const void* w_scales,
                                        const float* bias, void* y, int32_t y_type, int64_t ldy, int64_t M, int32_t N, int32_t K,
                                        void* workspace, size_t workspace_bytes, void* stream) {
    if (!gemm_sizes_ok(M, N, K) || !type_valid(x_type) || !type_valid(y_type)) return SPARQ_EINVAL;
    if (M == 0) return SPARQ_OK;
    if (!coded_ok(w_codes, w_scales) || !aligned(bias, 4)) return SPARQ_EINVAL;
    if (!tensor_ok(x, x_type, ldx, K) || !extent_ok(M, ldx) || !tensor_ok(y, y_type, ldy, N) || !extent_ok(M, ldy) || !extent_ok(M, K))
        return SPARQ_EINVAL;
    if (!workspace || !aligned(workspace, 256)) return SPARQ_EINVAL;
    if (workspace_bytes < coded_bytes(M, K)) return SPARQ_EWORKSPACE;
    if (M > 65535 * 64ll) return SPARQ_EUNSUPPORTED;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t *codes = static_cast<uint8_t*>(workspace), *scales = codes + round_up(M * code_pitch(K, 4), 256);
    const sparq_status q = launch_quantize(x, x_type, ldx, M, K, codes, scales, nullptr, nullptr, s);
    if (q != SPARQ_OK) return q;
    const GemmParams p = {codes, scales, static_cast<const uint8_t*>(w_codes), static_cast<const uint8_t*>(w_scales), bias, M, ldy,
                          code_pitch(K, 4), scale_pitch(K), N, (K + 63) / 64};
    return launch_gemm(p, y, y_type, s);
}
