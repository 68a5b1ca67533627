// Implemented in sparq_mx_few.hip: the product for at most kFewMost rows of codes, or kFewRows rows quantised on the way.
#pragma once
#include "sparq_mx_few_kernel.h"

namespace sparq {
namespace mx {

constexpr int kFewMost = 64;
sparq_status launch_few_rows(const FewParams& p, int x_type, void* y, int y_type, hipStream_t stream);

}  // namespace mx
}  // namespace sparq
