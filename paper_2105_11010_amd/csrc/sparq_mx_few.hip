#include "sparq_mx_few.h"

namespace sparq {
namespace mx {

template <class O, class X, int MT, int WAVES>
static void launch(const FewParams& p, void* y, hipStream_t stream) {
    few_rows_kernel<O, X, MT, WAVES><<<(p.N + kFewRows - 1) / kFewRows, WAVES * 64, few_lds_bytes<WAVES, MT>(p.M, p.x != nullptr), stream>>>(
        static_cast<O*>(y), p);
}
template <class O, class X, int MT>
static void launch_waves(const FewParams& p, void* y, hipStream_t stream) {
    // A wavefront a group up to eight of them (sixteen: 1 x 2048 x 8192 5.4 -> 6.1 us, 4 x 4096 x 8192 7.7 -> 7.4).
    if (p.groups <= 4) launch<O, X, MT, 4>(p, y, stream);
    else launch<O, X, MT, 8>(p, y, stream);
}

sparq_status launch_few_rows(const FewParams& p, int x_type, void* y, int y_type, hipStream_t stream) {
    with_type(y_type, [&](auto o) {
        typedef decltype(o) O;
        if (p.x) with_type(x_type, [&](auto x) { launch_waves<O, decltype(x), 1>(p, y, stream); });
        else if (p.M <= 16) launch_waves<O, void, 1>(p, y, stream);
        else if (p.M <= 32) launch_waves<O, void, 2>(p, y, stream);
        else if (p.M <= 48) launch_waves<O, void, 3>(p, y, stream);
        else launch_waves<O, void, 4>(p, y, stream);
    });
    return launch_status();
}

}  // namespace mx
}  // namespace sparq
