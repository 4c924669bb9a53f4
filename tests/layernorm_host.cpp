// Layer norm's host side for the CPU: what it would launch is written down instead.
#include <string.h>

#include <map>
#include <string>
#include <vector>

#include "k_layernorm.hip"

namespace {
struct Launch {
    uint32_t grid[3], block[3];
    unsigned char args[sizeof(co3_layernorm_backward_args)];   // the kernel's first argument
};
std::vector<Launch> launches;
dim3 next_grid, next_block;
size_t bytes;   // of the kernels' first argument
std::map<const void *, std::string> &kernels()   // those not launched yet; made before any other object here
{
    static std::map<const void *, std::string> m;
    return m;
}
}  // namespace

// What the compiler makes of a launch.
extern "C" {
char __hip_fatbin[1];
void **__hipRegisterFatBinary(const void *) { return nullptr; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *kernel, char *, const char *name, unsigned, uint3 *, uint3 *, dim3 *, dim3 *, int *)
{
    kernels()[kernel] = name;
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t)
{
    next_grid = grid;
    next_block = block;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream)
{
    *grid = next_grid;
    *block = next_block;
    *lds = 0;
    *stream = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *kernel, dim3 grid, dim3 block, void **args, size_t, hipStream_t)
{
    Launch l = {{grid.x, grid.y, grid.z}, {block.x, block.y, block.z}, {}};
    memcpy(l.args, args[0], bytes);
    launches.push_back(l);
    kernels().erase(kernel);
    return hipSuccess;
}
uint32_t not_launched() { return (uint32_t)kernels().size(); }
const char *one_not_launched() { return kernels().begin()->second.c_str(); }
hipError_t hipGetLastError() { return hipSuccess; }

// The launches of a call, at most `room` of them: their sizes, and the kernels' first arguments one behind the other.
static uint32_t put(Launch *out, uint32_t room)
{
    for (size_t k = 0; k < launches.size() && k < room; ++k) out[k] = launches[k];
    return (uint32_t)launches.size();
}
uint32_t forward_launches(const co3_layernorm_args *a, Launch *out, uint32_t room)
{
    launches.clear();
    bytes = sizeof(*a);
    (void)co3::launch_layernorm(*a, nullptr);
    return put(out, room);
}
size_t backward_workspace(uint32_t U, uint64_t rows, uint32_t cols) { return co3::layernorm_backward_workspace_bytes(U, rows, cols); }
uint32_t backward_launches(const co3_layernorm_backward_args *a, Launch *out, uint32_t room)
{
    launches.clear();
    bytes = sizeof(*a);
    (void)co3::launch_layernorm_backward(*a, nullptr);
    return put(out, room);
}
}

namespace co3 {
ProfScope::ProfScope(int, hipStream_t) {}
ProfScope::~ProfScope() {}
}  // namespace co3
