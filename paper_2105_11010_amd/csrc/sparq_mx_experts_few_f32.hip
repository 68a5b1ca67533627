#include "sparq_mx_experts_gemm.h"

namespace sparq {
namespace mx {
sparq_status launch_experts_few_f32(const ExpertFewParams& p, int x_type, int fragments, int64_t pieces, void* y, hipStream_t stream) {
    return launch_experts_few<float>(p, x_type, fragments, pieces, y, stream);
}
}  // namespace mx
}  // namespace sparq
