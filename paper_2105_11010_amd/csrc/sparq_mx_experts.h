// What the operators of a block with experts share (include/sparq_mx_experts.h).
#pragma once
#include "../../include/sparq_mx_experts.h"
#include "sparq_mx_common.h"

namespace sparq {
namespace mx {

inline bool experts_ok(int experts) { return experts >= 1; }

#if defined(__HIPCC__)
// Eight elements as they lie in memory, of which the first n are there (zeros for the others).
template <bool NT, class T>
__device__ __forceinline__ void load_raw_upto8(const T* p, int n, Raw8<T>& r) {
    if (n >= 8) {
        load_raw<NT>(p, r);
        return;
    }
    r = Raw8<T>{};
    if (n > 0) {
        typedef std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t> Bits;
        Bits e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = reinterpret_cast<const Bits*>(p)[i < n ? i : 0];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t v = i < n ? e[i] : (Bits)0;
            if constexpr (sizeof(T) == 4) r.w[i] = v;
            else r.w[i >> 1] |= v << (16 * (i & 1));
        }
    }
}
template <bool NT, class T>
__device__ __forceinline__ void store_raw_upto8(T* p, int n, const Raw8<T>& r) {
    if (n >= 8) {
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) word_to<NT>(p + 4 * h, v4u{r.w[4 * h], r.w[4 * h + 1], r.w[4 * h + 2], r.w[4 * h + 3]});
        return;
    }
    typedef std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t> Bits;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) reinterpret_cast<Bits*>(p)[i] = sizeof(T) == 4 ? (Bits)r.w[i] : (Bits)(r.w[i >> 1] >> (16 * (i & 1)));
}
#endif

}  // namespace mx
}  // namespace sparq
