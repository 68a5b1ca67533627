// Layer norm with an 8-bit checkpoint of its input, and its backward pass from that (include/sparq_mx.h).
#include <type_traits>

#include "sparq_mx_common.h"

namespace sparq {
namespace mx {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

struct NormParams {
    int64_t ldx, ldy, code_pitch, scale_pitch, rows;
    int32_t K, K128;
    float eps, inv_K;
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}
// Sum over the wavefronts that share a row.  Two buffers in turn: a wavefront may write the next sum while others still
// read this one, but not the one after that before they have passed the barrier between.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float* shared, int& turn) {
    v = wave_sum(v);
    if constexpr (WAVES == 1) return v;
    float* at = shared + turn * WAVES;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = at[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) s += at[i];
    return s;
}
__device__ __forceinline__ void load_upto8_f32(const float* p, int n, float (&v)[8]) {
    if (n > 0) load_upto8(p, n, v);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    }
}

// WAVES wavefronts take a row, CHUNKS x 8 values a lane, which stay in registers from the load to the result: one pass over
// memory, the mean first and the squares of what differs from it second.  CHUNKS 0: rows of any length, read three times.
template <class T, int WAVES, int CHUNKS>
__global__ __launch_bounds__(kThreads) void norm_kernel(const T* __restrict__ x, const float* __restrict__ gamma,
                                                        const float* __restrict__ beta, T* __restrict__ y, float* __restrict__ mean_out,
                                                        float* __restrict__ rstd_out, uint8_t* __restrict__ codes,
                                                        uint8_t* __restrict__ scales, const NormParams p) {
    __shared__ float shared[2 * WAVES];
    constexpr int kPerBlock = kWaves / WAVES, kSpan = WAVES * 64 * 8;
    const int wave = threadIdx.x >> 6, t = threadIdx.x & (WAVES * 64 - 1), lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * kPerBlock + (WAVES == 1 ? wave : 0);
    if (row >= p.rows) return;                               // (whole workgroups where they share a row)
    int turn = 0;
    x += row * p.ldx;
    y += row * p.ldy;
    const int chunks = CHUNKS ? CHUNKS : (int)((p.K + kSpan - 1) / kSpan);
    constexpr int kHeld = CHUNKS ? CHUNKS : 1;
    float v[kHeld][8];
    float sum = 0.0f;
    auto fetch = [&](int c) __attribute__((always_inline)) {
        const int col = c * kSpan + 8 * t;
        if (col < p.K) load_upto8(x + col, p.K - col, v[CHUNKS ? c : 0]);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[CHUNKS ? c : 0][i] = 0.0f;
        }
    };
    if constexpr (CHUNKS > 0) {                              // all of them on their way before the first is used
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) fetch(c);
    }
#pragma unroll kHeld
    for (int c = 0; c < chunks; ++c) {
        if constexpr (CHUNKS == 0) fetch(c);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += v[CHUNKS ? c : 0][i];
    }
    const float mean = row_sum<WAVES>(sum, shared, turn) * p.inv_K;
    float squares = 0.0f;
#pragma unroll kHeld
    for (int c = 0; c < chunks; ++c) {
        if constexpr (CHUNKS == 0) fetch(c);
        const int n = p.K - (c * kSpan + 8 * t);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = v[CHUNKS ? c : 0][i] - mean;
            squares += i < n ? d * d : 0.0f;
        }
    }
    const float var = row_sum<WAVES>(squares, shared, turn) * p.inv_K;
    const float rstd = 1.0f / sqrtf(var + p.eps);
    if (t == 0 && mean_out) mean_out[row] = mean;
    if (t == 0 && rstd_out) rstd_out[row] = rstd;
#pragma unroll kHeld
    for (int c = 0; c < chunks; ++c) {
        if constexpr (CHUNKS == 0) fetch(c);
        const int col = c * kSpan + 8 * t, n = p.K - col;
        float g[8], b[8], o[8];
        load_upto8_f32(gamma + col, n, g);
        if (beta) load_upto8_f32(beta + col, n, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (v[CHUNKS ? c : 0][i] - mean) * rstd * g[i] + (beta ? b[i] : 0.0f);
        if (n > 0) store_upto8(y + col, n, o);
        if (codes && col - 8 * lane < p.K) {                 // the wavefront's 512 values begin inside the row
            const uint32_t byte = scale8_of(block_top(v[CHUNKS ? c : 0]));
            const v2u w = codes8_of(v[CHUNKS ? c : 0], byte);
            if (col < p.K128) *reinterpret_cast<v2u*>(codes + row * p.code_pitch + col) = w;
            if ((lane & 3) == 0) scales[row * p.scale_pitch + (col >> 5)] = (uint8_t)byte;
        }
    }
}

// ---- backward ----------------------------------------------------------------------
struct NormGradParams {
    int64_t ldy, ldx, code_pitch, scale_pitch, rows;
    int32_t K;
    float inv_K;
    int32_t parts;                       // partial sums of the weights' gradients: rows part, part + parts, ...
};

// Row sums of d and d h (d = dy gamma, h = (X - mean) rstd), one wavefront a row.
template <class T>
__global__ __launch_bounds__(kThreads) void norm_grad_rows_kernel(const T* __restrict__ dy, const uint8_t* __restrict__ codes,
                                                                  const uint8_t* __restrict__ scales, const float* __restrict__ mean,
                                                                  const float* __restrict__ rstd, const float* __restrict__ gamma,
                                                                  v2f* __restrict__ sums, const NormGradParams p) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (row >= p.rows) return;
    const float mu = mean[row], r = rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int col = 8 * lane; col < p.K; col += 512) {
        const int n = p.K - col;
        float d[8], h[8], g[8];
        load_upto8(dy + row * p.ldy + col, n, d);
        load_upto8(gamma + col, n, g);
        values8_of(*reinterpret_cast<const v2u*>(codes + row * p.code_pitch + col), scales[row * p.scale_pitch + (col >> 5)], h);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float e = d[i] * g[i];                     // (zero past the row)
            s1 += e;
            s2 += e * ((h[i] - mu) * r);
        }
    }
    s1 = wave_sum(s1);
    s2 = wave_sum(s2);
    if (lane == 0) sums[row] = v2f{s1 * p.inv_K, s2 * p.inv_K};
}

// dx, and this workgroup's share of the weights' gradients: 2048 columns of rows part, part + parts, ...
template <class T>
__global__ __launch_bounds__(kThreads) void norm_grad_columns_kernel(const T* __restrict__ dy, const uint8_t* __restrict__ codes,
                                                                     const uint8_t* __restrict__ scales, const float* __restrict__ mean,
                                                                     const float* __restrict__ rstd, const float* __restrict__ gamma,
                                                                     const v2f* __restrict__ sums, T* __restrict__ dx,
                                                                     float* __restrict__ partial, const NormGradParams p) {
    const int col = (blockIdx.x * kThreads + threadIdx.x) * 8, n = p.K - col;
    if (n <= 0) return;
    float g[8], dg[8] = {}, db[8] = {};
    load_upto8(gamma + col, n, g);
    for (int64_t row = blockIdx.y; row < p.rows; row += p.parts) {
        const float mu = mean[row], r = rstd[row];
        const v2f s = sums[row];
        float d[8], h[8], o[8];
        load_upto8(dy + row * p.ldy + col, n, d);
        values8_of(*reinterpret_cast<const v2u*>(codes + row * p.code_pitch + col), scales[row * p.scale_pitch + (col >> 5)], h);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float hh = (h[i] - mu) * r;
            o[i] = r * (d[i] * g[i] - s[0] - hh * s[1]);
            dg[i] += d[i] * hh;
            db[i] += d[i];
        }
        store_upto8(dx + row * p.ldx + col, n, o);
    }
    if (partial) {
        float* at = partial + (int64_t)blockIdx.y * 2 * p.K + col;
        store_upto8(at, n, dg);
        store_upto8(at + p.K, n, db);
    }
}

// The partial sums' sum, part after part.
__global__ __launch_bounds__(kThreads) void norm_grad_join_kernel(const float* __restrict__ partial, float* __restrict__ dgamma,
                                                                  float* __restrict__ dbeta, int K, int parts) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= 2 * K) return;
    float* out = c < K ? dgamma : dbeta;
    if (!out) return;
    float s = 0.0f;
    for (int i = 0; i < parts; ++i) s += partial[(int64_t)i * 2 * K + c];
    out[c < K ? c : c - K] = s;
}

static int norm_parts(int64_t rows) { return (int)(rows < 256 ? rows : 256); }
static size_t norm_grad_bytes(int64_t rows, int K) {
    return (size_t)(round_up(rows * 8, 256) + round_up((int64_t)norm_parts(rows) * 2 * K * 4, 256));
}

}  // namespace mx
}  // namespace sparq

using namespace sparq;
using namespace sparq::mx;

extern "C" sparq_status sparq_mx_norm(const void* x, int64_t ldx, const float* gamma, const float* beta, float eps, void* y, int64_t ldy,
                                      int32_t type, float* mean, float* rstd, void* codes, void* scales, int64_t rows, int32_t K,
                                      void* stream) {
    if (!sizes_ok(rows, K) || !type_valid(type) || !(eps >= 0.0f)) return SPARQ_EINVAL;
    if (rows == 0) return SPARQ_OK;
    if (!tensor_ok(x, type, ldx, K) || !tensor_ok(y, type, ldy, K) || !gamma || !aligned(gamma, 4) || !aligned(beta, 4)) return SPARQ_EINVAL;
    if (!extent_ok(rows, ldx) || !extent_ok(rows, ldy) || !extent_ok(rows, K) || !coded_ok_or_none(codes, scales)) return SPARQ_EINVAL;
    if ((mean != nullptr) != (rstd != nullptr) || !aligned(mean, 4) || !aligned(rstd, 4)) return SPARQ_EINVAL;
    if (rows >= (1ll << 31)) return SPARQ_EUNSUPPORTED;
    const NormParams p = {ldx, ldy, code_pitch(K, 8), scale_pitch(K), rows, K, (int)round_up(K, kCodeUnit), eps, (float)(1.0 / K)};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const auto launch = [&](auto kernel, int per_block) {
            kernel<<<(unsigned)((rows + per_block - 1) / per_block), kThreads, 0, s>>>(
                static_cast<const T*>(x), gamma, beta, static_cast<T*>(y), mean, rstd, static_cast<uint8_t*>(codes),
                static_cast<uint8_t*>(scales), p);
        };
        if (K <= 512) launch(norm_kernel<T, 1, 1>, 4);
        else if (K <= 1024) launch(norm_kernel<T, 1, 2>, 4);
        else if (K <= 2048) launch(norm_kernel<T, 4, 1>, 1);
        else if (K <= 4096) launch(norm_kernel<T, 4, 2>, 1);
        else if (K <= 8192) launch(norm_kernel<T, 4, 4>, 1);
        else launch(norm_kernel<T, 4, 0>, 1);
    });
    return launch_status();
}

extern "C" size_t sparq_mx_norm_grad_workspace_bytes(int64_t rows, int32_t K) {
    return sizes_ok(rows, K) && extent_ok(rows, K) ? norm_grad_bytes(rows, K) : 0;
}

extern "C" sparq_status sparq_mx_norm_grad(const void* dy, int64_t lddy, const void* codes, const void* scales, const float* mean,
                                           const float* rstd, const float* gamma, void* dx, int64_t lddx, int32_t type, float* dgamma,
                                           float* dbeta, int64_t rows, int32_t K, void* workspace, size_t workspace_bytes, void* stream) {
    if (!sizes_ok(rows, K) || !type_valid(type) || !aligned(dgamma, 4) || !aligned(dbeta, 4)) return SPARQ_EINVAL;
    if (!extent_ok(rows, K)) return SPARQ_EINVAL;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const unsigned join = (unsigned)((2ll * K + kThreads - 1) / kThreads);
    if (rows == 0) {
        if (dgamma || dbeta) norm_grad_join_kernel<<<join, kThreads, 0, s>>>(nullptr, dgamma, dbeta, K, 0);
        return launch_status();
    }
    if (!tensor_ok(dy, type, lddy, K) || !tensor_ok(dx, type, lddx, K) || !coded_ok(codes, scales)) return SPARQ_EINVAL;
    if (!mean || !rstd || !gamma || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(gamma, 4)) return SPARQ_EINVAL;
    if (!extent_ok(rows, lddy) || !extent_ok(rows, lddx)) return SPARQ_EINVAL;
    if (rows >= (1ll << 31)) return SPARQ_EUNSUPPORTED;
    if (!workspace || !aligned(workspace, 256)) return SPARQ_EINVAL;
    if (workspace_bytes < norm_grad_bytes(rows, K)) return SPARQ_EWORKSPACE;
    v2f* sums = static_cast<v2f*>(workspace);
    float* partial = dgamma || dbeta ? reinterpret_cast<float*>(static_cast<char*>(workspace) + round_up(rows * 8, 256)) : nullptr;
    const NormGradParams p = {lddy, lddx, code_pitch(K, 8), scale_pitch(K), rows, K, (float)(1.0 / K), norm_parts(rows)};
    const uint8_t *c = static_cast<const uint8_t*>(codes), *sc = static_cast<const uint8_t*>(scales);
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        norm_grad_rows_kernel<T><<<(unsigned)((rows + kWaves - 1) / kWaves), kThreads, 0, s>>>(
            static_cast<const T*>(dy), c, sc, mean, rstd, gamma, sums, p);
        norm_grad_columns_kernel<T><<<dim3((unsigned)((K + 8ll * kThreads - 1) / (8 * kThreads)), p.parts), kThreads, 0, s>>>(
            static_cast<const T*>(dy), c, sc, mean, rstd, gamma, sums, static_cast<T*>(dx), partial, p);
    });
    if (partial) norm_grad_join_kernel<<<join, kThreads, 0, s>>>(partial, dgamma, dbeta, K, p.parts);
    return launch_status();
}
