// Loads from memory to LDS without a register in between, and the meetings of a workgroup that do not wait for them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace co3 {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 64 lanes' 16 bytes: from base + offset (of every lane) + k, to `lds` + 16 lane; zeros where offset + k is not within the buffer.
// Written out, since the compiler would wait for all loads to LDS before every read of LDS.  Who reads waits with wait_loads().
// m0 is named for the compiler's own writes to it; no value lives there, which is what its warning is about.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void load_to_lds(u32x4 base, uint32_t offset, uint32_t k, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "s"(lds), "v"(offset), "s"(base), "s"(k) : "m0", "memory");
}
// 64 lanes' four bytes, to `lds` + 4 lane.
__device__ inline void load_word_to_lds(u32x4 base, uint32_t offset, uint32_t k, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" : : "s"(lds), "v"(offset), "s"(base), "s"(k) : "m0", "memory");
}
#pragma clang diagnostic pop

// Until all but the wavefront's last `left` loads are there.
template <int left>
__device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(left) : "memory"); }

// All wavefronts of the workgroup, each with what it asked of LDS.  (__syncthreads() would wait for the loads to LDS as well.)
__device__ inline void meet()
{
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}

// A buffer of `bytes` from p on, for load_to_lds.
__device__ inline u32x4 buffer_of(const void *p, uint32_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    u32x4 r = {(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, bytes, 0x00027000u};
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (uint32_t)__builtin_amdgcn_readfirstlane((int)r[i]);
    return r;
}

}  // namespace co3
