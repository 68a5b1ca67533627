#include "sparq_mx_few.h"

namespace sparq {
namespace mx {

template <class O, class X, int MT, int WAVES>
static sparq_status launch(const FewParams& p, void* y, hipStream_t stream) {
    return in_launches((p.N + kFewRows - 1) / kFewRows, WAVES * 64, [&](int64_t first, int64_t n) {
        FewParams q = p;                                     // of the columns from here on
        const int64_t column = first * kFewRows;
        q.w += column * p.code_pitch;
        q.ws += column * p.scale_pitch;
        if (q.bias) q.bias += column;
        q.N -= (int)column;
        few_rows_kernel<O, X, MT, WAVES><<<(unsigned)n, WAVES * 64, few_lds_bytes<WAVES, MT>(p.M, p.x != nullptr), stream>>>(static_cast<O*>(y) + column, q);
        return launch_status();
    });
}
template <class O, class X, int MT>
static sparq_status launch_waves(const FewParams& p, void* y, hipStream_t stream) {
    // A wavefront a group up to eight of them (sixteen: 1 x 2048 x 8192 5.4 -> 6.1 us, 4 x 4096 x 8192 7.7 -> 7.4).
    return p.groups <= 4 ? launch<O, X, MT, 4>(p, y, stream) : launch<O, X, MT, 8>(p, y, stream);
}

sparq_status launch_few_rows(const FewParams& p, int x_type, void* y, int y_type, hipStream_t stream) {
    sparq_status s = SPARQ_OK;
    with_type(y_type, [&](auto o) {
        typedef decltype(o) O;
        if (p.x) with_type(x_type, [&](auto x) { s = launch_waves<O, decltype(x), 1>(p, y, stream); });
        else if (p.M <= 16) s = launch_waves<O, void, 1>(p, y, stream);
        else if (p.M <= 32) s = launch_waves<O, void, 2>(p, y, stream);
        else if (p.M <= 48) s = launch_waves<O, void, 3>(p, y, stream);
        else s = launch_waves<O, void, 4>(p, y, stream);
    });
    return s;
}

}  // namespace mx
}  // namespace sparq
