// The tensor types of the training operators, CO3_F32, CO3_BF16 and CO3_F16, and loads of up to 16 bytes of them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "co3.h"

namespace co3 {

inline size_t type_bytes(int32_t type) { return type == CO3_F32 ? 4 : 2; }

// N elements next to each other.  Rows may begin at any element, so the vector asks for no more than an element's alignment;
// the GPU loads and stores 16 bytes at any address all the same.
template <typename T, int N> struct Pack;
template <int N> struct Pack<float, N> { typedef float V __attribute__((ext_vector_type(N), aligned(4))); };
template <int N> struct Pack<__bf16, N> { typedef __bf16 V __attribute__((ext_vector_type(N), aligned(2))); };
template <int N> struct Pack<_Float16, N> { typedef _Float16 V __attribute__((ext_vector_type(N), aligned(2))); };
template <typename T> constexpr int kVec = 16 / (int)sizeof(T);   // elements of 16 bytes

// v[i] = p[i] for i < n; the others are `fill`.  n <= 0: nothing is read.
template <typename T, int N>
__device__ inline typename Pack<T, N>::V load_pack(const T *p, int n, T fill = (T)0.f)
{
    typename Pack<T, N>::V v;
    if (n >= N) {
        v = *reinterpret_cast<const typename Pack<T, N>::V *>(p);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = fill;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) v[i] = p[i];
    }
    return v;
}

template <typename T, int N>
__device__ inline void store_pack(T *p, int n, const typename Pack<T, N>::V &v)
{
    if (n >= N) {
        *reinterpret_cast<typename Pack<T, N>::V *>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) p[i] = v[i];
    }
}

}  // namespace co3
