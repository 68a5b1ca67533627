// The activations and their slopes.
#pragma once
#include "sparq_mx_common.h"

namespace sparq {
namespace mx {

// f(v) and f'(v).  PRECISE (fp32 tensors): the library's exponential, erfc and division; else the instructions' (2 and 1 ulp of fp32) and the
// approximation below, whose errors are relative ones far below what a 16-bit result keeps, below 0 as well, where f is all tail.
template <bool PRECISE>
__device__ __forceinline__ float sigmoid(float v) {
    if constexpr (PRECISE) return 1.0f / (1.0f + expf(-v));
    else return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.44269504f));
}
// The normal distribution's integral and exp(-v^2 / 2), for 16-bit results.  Below 0 the integral is that exponential times a function that
// falls like 1 / |v|: t p(t), t = 1 / (1 + 0.264 |v|), p fitted to the least largest relative error for |v| up to 13.5 (beyond, the exponential is
// zero), 5.4e-7.  With fp32's roundings, most of them of v^2 in the exponent, the integral is off by at most (32 + 2 v^2) 2^-24 of itself.
__device__ __forceinline__ float normal_integral(float v, float& density) {
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.264f * __builtin_fabsf(v));
    density = __builtin_amdgcn_exp2f(v * v * -0.721347520f);
    const float p = 0.10517378f + t * (0.10781906f + t * (0.08047569f + t * (0.14862743f + t * (-0.076199844f + t * (0.20336618f + t * -0.06926256f)))));
    const float tail = t * p * density;
    return v < 0.0f ? tail : 1.0f - tail;
}
template <int F, bool PRECISE>
__device__ __forceinline__ float function(float v) {
    float density;
    if constexpr (F == SPARQ_MX_SILU) return v * sigmoid<PRECISE>(v);
    else if constexpr (PRECISE) return 0.5f * v * erfcf(v * -0.707106781f);
    else return v * normal_integral(v, density);
}
template <int F, bool PRECISE>
__device__ __forceinline__ void function_and_slope(float v, float& value, float& slope) {
    if constexpr (F == SPARQ_MX_SILU) {
        const float s = sigmoid<PRECISE>(v);
        value = v * s;
        slope = s + value * (1.0f - s);
    } else {
        float density;
        const float c = PRECISE ? 0.5f * erfcf(v * -0.707106781f) : normal_integral(v, density);
        if (PRECISE) density = expf(-0.5f * v * v);
        value = v * c;
        slope = c + v * (0.398942280f * density);
    }
}

}  // namespace mx
}  // namespace sparq
