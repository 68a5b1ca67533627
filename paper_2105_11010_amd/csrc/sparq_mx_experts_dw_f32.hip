#include "sparq_mx_experts_grad.h"

namespace sparq {
namespace mx {
sparq_status launch_experts_dw_f32(const ExpertGradParams& p, dim3 grid, int tile, void* out, bool f32, hipStream_t stream) {
    return launch_experts_grad<float, true>(p, grid, tile, out, f32, stream);
}
}  // namespace mx
}  // namespace sparq
