// What the kernels of the Newton-Schulz iteration share (k_ortho.hip, k_ortho_small.hip).
#pragma once

#include "ortho.h"
#include "tensor_types.h"

namespace co3 {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr float kScaleX = 16384.f, kScaleB = 8192.f;   // 2^14, also of A; 2^13

struct Polynomial { float a, b, c; };

__device__ inline void split(float v, _Float16 &hi, _Float16 &lo)
{
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// 2^14 / (norm + eps) of a sum of squares: 0 for a matrix of zeros, NaN for one that is not finite.
__device__ inline double scale_of(double squares, float eps)
{
    const bool finite = squares < INFINITY;   // false for NaN too
    return !finite ? (double)NAN : squares > 0.0 ? (double)kScaleX / (sqrt(squares) + (double)eps) : 0.0;
}
__device__ inline void count_not_finite(const OrthoCall &c)
{
    if (c.status) atomicAdd(reinterpret_cast<unsigned long long *>(c.status + CO3_STAT_NONFINITE), 1ull);
}

// Eight results next to each other in a row of the caller's matrix.
__device__ inline void store_result(const OrthoLayout &lay, const OrthoCall &c, const MatDev &m, uint32_t r, uint32_t col, const float *v)
{
    if (r >= m.rows || col >= m.cols) return;
    const int n = (int)(m.cols - col);
    const uint64_t at = m.offset + (uint64_t)r * m.ld + col;
    const float scale = m.scale / kScaleX;
    if (!c.out) {
        const float keep = 1.f - c.eta * c.decay, step = c.eta * scale;
        auto w = load_pack<float, 8>(c.model + at, n);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = w[i] * keep - step * v[i];
        store_pack<float, 8>(c.model + at, n, w);
    } else if (lay.type == CO3_F32) {
        Pack<float, 8>::V o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = v[i] * scale;
        store_pack<float, 8>(static_cast<float *>(c.out) + at, n, o);
    } else if (lay.type == CO3_BF16) {
        Pack<__bf16, 8>::V o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (__bf16)(v[i] * scale);
        store_pack<__bf16, 8>(static_cast<__bf16 *>(c.out) + at, n, o);
    } else {
        Pack<_Float16, 8>::V o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (_Float16)(v[i] * scale);
        store_pack<_Float16, 8>(static_cast<_Float16 *>(c.out) + at, n, o);
    }
}

}  // namespace co3
