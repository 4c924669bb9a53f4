// Group norm's backward pass from x as it is (groupnorm_backward.h).
#include "groupnorm_backward.h"

namespace co3 {

hipError_t launch_groupnorm_backward8(const co3_groupnorm_backward_args &a, hipStream_t s);   // k_groupnorm_backward8.hip

hipError_t launch_groupnorm_backward(const co3_groupnorm_backward_args &a, hipStream_t s)
{
    return a.x ? launch_backward<false>(a, s) : launch_groupnorm_backward8(a, s);
}

}  // namespace co3
