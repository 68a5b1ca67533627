#include "sparq_mx_experts_gemm.h"

namespace sparq {
namespace mx {
sparq_status launch_experts_tiles_f16(const ExpertGemmParams& p, int tile, void* y, hipStream_t stream) { return launch_experts_tiles<_Float16>(p, tile, y, stream); }
}  // namespace mx
}  // namespace sparq
