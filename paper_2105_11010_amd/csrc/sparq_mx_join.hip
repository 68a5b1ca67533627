// Where a reduction was divided among workgroups: the parts' sum.
#include "sparq_mx_common.h"

namespace sparq {
namespace mx {

constexpr int kThreads = 256;

// out = the parts' sum, part after part; four values a thread.
template <class O>
__global__ __launch_bounds__(kThreads) void join_kernel(const float* __restrict__ partial, const float* __restrict__ bias, O* __restrict__ out,
                                                        int64_t J, int K, int64_t ldo, int parts) {
    const int k = (blockIdx.x * kThreads + threadIdx.x) * 4;
    if (k >= K) return;
    const int n = K - k < 4 ? K - k : 4;
    const bool words = K % 4 == 0;                           // (rows of partial results are K apart)
    float b[4] = {};
    if (bias) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) b[e] = bias[k + e];
    }
    for (int64_t j = blockIdx.y; j < J; j += gridDim.y) {
        v4f s = {};
        const float* at = partial + j * K + k;
        for (int i = 0; i < parts; ++i, at += J * K) {
            if (words) s += *reinterpret_cast<const v4f*>(at);
            else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < n) s[e] += at[e];
            }
        }
        O* to = out + j * ldo + k;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) to[e] = (O)(s[e] + b[e]);
    }
}

sparq_status launch_join(const float* partial, const float* bias, void* out, int type, int64_t J, int K, int64_t ldo, int parts, hipStream_t stream) {
    const unsigned gx = (unsigned)((K + 4ll * kThreads - 1) / (4 * kThreads));
    with_type(type, [&](auto o) {
        typedef decltype(o) O;
        join_kernel<O><<<dim3(gx, (unsigned)(J < 65535 ? J : 65535)), kThreads, 0, stream>>>(partial, bias, static_cast<O*>(out), J, K, ldo, parts);
    });
    return launch_status();
}

// Sums over rows, few columns of many parts: 32 columns a workgroup (from column `from` on), every 32nd part a thread, joined in LDS.
constexpr int kJoinThreads = 1024;
__global__ __launch_bounds__(kJoinThreads) void join_columns_kernel(const float* __restrict__ partial, float* __restrict__ first,
                                                                    float* __restrict__ second, int split, int columns, int parts, int from) {
    __shared__ float shared[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = from + blockIdx.x * 32 + x;
    float s = 0.0f;
    if (c < columns) {
#pragma unroll 4
        for (int i = y; i < parts; i += 32) s += partial[(int64_t)i * columns + c];
    }
    shared[y][x] = s;
    __syncthreads();
    if (y != 0 || c >= columns) return;
#pragma unroll
    for (int i = 1; i < 32; ++i) s += shared[i][x];
    float* out = c < split ? first : second;
    if (out) out[c < split ? c : c - split] = s;
}
sparq_status launch_join_columns(const float* partial, float* first, float* second, int split, int columns, int parts, hipStream_t stream) {
    return in_launches((columns + 31ll) / 32, kJoinThreads, [&](int64_t at, int64_t n) {
        join_columns_kernel<<<(unsigned)n, kJoinThreads, 0, stream>>>(partial, first, second, split, columns, parts, (int)(32 * at));
        return launch_status();
    });
}

}  // namespace mx
}  // namespace sparq
