#include "sparq_mx_grad.h"

namespace sparq {
namespace mx {
sparq_status launch_grad_dx_bf16(const GradParams& p, int parts, int tile, void* out, int out_type, hipStream_t stream) {
    return launch_grad_types<__bf16, false>(p, parts, tile, out, out_type, stream);
}
}  // namespace mx
}  // namespace sparq
