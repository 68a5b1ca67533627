#include "sparq_mx_experts_gemm.h"

namespace sparq {
namespace mx {
sparq_status launch_experts_tiles_f32(const ExpertGemmParams& p, int tile, void* y, hipStream_t stream) { return launch_experts_tiles<float>(p, tile, y, stream); }
}  // namespace mx
}  // namespace sparq
