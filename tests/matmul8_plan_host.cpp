// The host side of the operators in 8 bits for the CPU: a launch does nothing, and how a product is cut can be asked for.
#include "co3_train8.cpp"

namespace co3 {
hipError_t launch_quantize8(const co3_quantize8_args &, hipStream_t) { return hipSuccess; }
hipError_t launch_dequantize8(const co3_dequantize8_args &, hipStream_t) { return hipSuccess; }
hipError_t launch_matmul8(const co3_matmul8_args &, const Matmul8Plan &, hipStream_t) { return hipSuccess; }
size_t groupnorm_workspace_bytes(uint64_t, uint64_t, uint32_t, uint32_t, int32_t) { return 0; }
size_t groupnorm_backward_workspace_bytes(uint32_t, uint64_t, uint64_t, uint32_t, uint32_t, int32_t) { return 0; }
hipError_t launch_groupnorm(const co3_groupnorm_args &, hipStream_t) { return hipSuccess; }
hipError_t launch_groupnorm_backward(const co3_groupnorm_backward_args &, hipStream_t) { return hipSuccess; }
}  // namespace co3

extern "C" int plan_of(const co3_matmul8_args *a, uint32_t *form, uint32_t *slices)
{
    Matmul8Plan p;
    const int rc = plan_matmul8(*a, &p);
    *form = p.form;
    *slices = p.slices;
    return rc;
}
