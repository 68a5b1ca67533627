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

}  // namespace mx
}  // namespace sparq
