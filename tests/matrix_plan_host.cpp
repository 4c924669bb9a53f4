// The host side of the training operators for the CPU: its calls of the device's memory go to the host's, and a launch does nothing.
#include <hip/hip_runtime.h>

#include <stdlib.h>
#include <string.h>

static hipError_t host_device(int *d) { *d = 0; return hipSuccess; }
static hipError_t host_malloc(void **p, size_t n) { *p = malloc(n); return *p ? hipSuccess : hipErrorOutOfMemory; }
static hipError_t host_copy(void *to, const void *from, size_t n, hipMemcpyKind) { memcpy(to, from, n); return hipSuccess; }
static hipError_t host_free(void *p) { free(p); return hipSuccess; }
#define hipGetDevice host_device
#define hipSetDevice(d) hipSuccess
#define hipMalloc host_malloc
#define hipMemcpy host_copy
#define hipFree host_free
#include "co3_train.cpp"

namespace co3 {
hipError_t launch_orthogonalize(const OrthoLayout &, const OrthoCall &, hipStream_t) { return hipSuccess; }
hipError_t launch_layernorm(const co3_layernorm_args &, hipStream_t) { return hipSuccess; }
size_t layernorm_backward_workspace_bytes(uint32_t, uint64_t, uint32_t) { return 0; }
hipError_t launch_layernorm_backward(const co3_layernorm_backward_args &, hipStream_t) { return hipSuccess; }
}  // namespace co3
