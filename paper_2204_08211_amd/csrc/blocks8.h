// Tensors of e4m3 numbers with a power of two for each block, as the kernels read them (co3_blocks8 of include/co3.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "co3.h"

namespace co3 {

constexpr uint32_t kBlockCols = 128;   // columns of a block

__host__ __device__ inline uint32_t block_columns(const co3_blocks8 &b) { return (b.cols + kBlockCols - 1) / kBlockCols; }
inline uint64_t block_rows_of(const co3_blocks8 &b) { return b.block_rows == 1 ? b.rows : (b.rows + 127) / 128; }

// 2^(byte - 127), byte >= 1
__device__ inline float power_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Four numbers of a word.
__device__ inline void numbers_of(uint32_t word, float *v)
{
    typedef float float2v __attribute__((ext_vector_type(2)));
    const float2v a = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, true);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
}

}  // namespace co3
