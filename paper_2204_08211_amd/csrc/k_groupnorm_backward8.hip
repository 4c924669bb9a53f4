// Group norm's backward pass from x kept in 8 bits (groupnorm_backward.h).
#include "groupnorm_backward.h"

namespace co3 {

hipError_t launch_groupnorm_backward8(const co3_groupnorm_backward_args &a, hipStream_t s) { return launch_backward<true>(a, s); }

}  // namespace co3
