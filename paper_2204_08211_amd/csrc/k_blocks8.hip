// To 8 bits and back: e4m3 numbers with a power of two for each block of 128 columns by 128 rows or by one.
//
// A block's exponent e is the least (-126 at least) with max |x| <= 448 2^e; a value is x 2^-e rounded to e4m3.  Scaling by a power
// of two rounds nothing, so a number is rounded once, and the same number has the same bytes whoever scales it.  The precision of a
// floating-point format does not depend on the scale: a power of two loses no more than half of the 2^15 that lie between the largest
// number and the smallest one of full precision.
// Both are bound by memory.  A block stays in registers between its largest value and its bytes.
// Measured (MI355X, a large copy runs at 4.8 TB/s; kernels): 4 x 4096 x 4096 bf16 to 8 bits 47 to 52 us = 4.3 to 3.9 TB/s, and back 37 us = 5.4 TB/s, right behind
// it; 64 x 257, 5.1 and 3.7 us, a launch.
#include "blocks8.h"
#include "co3_internal.h"
#include "tensor_types.h"

namespace co3 {

// Exponent + 127 of a block whose largest finite value is m.
__device__ inline uint32_t scale_byte(float m)
{
    if (m == 0.f) return 127;
    const uint32_t bits = __float_as_uint(m), field = bits >> 23;   // m < 2^-126: field 0, far below 1 in any case
    const int e = (int)field - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);   // m = f 2^(field - 127), 448 = 1.75 2^8
    return e < 1 ? 1u : (uint32_t)e;
}

__device__ inline float finite_size(float v)
{
    const float a = fabsf(v);
    return a < INFINITY ? a : 0.f;   // false for NaN too
}

// Sixteen values' bytes.  `odd`: some are not finite; they become the NaN without a sign.
__device__ inline uint4 bytes_of(const float (&v)[16], float inverse, bool odd)
{
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        int word = 0;
        word = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * q] * inverse, v[4 * q + 1] * inverse, word, false);
        word = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * q + 2] * inverse, v[4 * q + 3] * inverse, word, true);
        w[q] = (uint32_t)word;
    }
    if (odd) {
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i / 4] = fabsf(v[i]) < INFINITY ? w[i / 4] : (w[i / 4] & ~(0xffu << (i % 4 * 8))) | 0x7fu << (i % 4 * 8);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T> struct Sixteen { typename Pack<T, kVec<T>>::V p[16 / kVec<T>]; };

template <typename T>
__device__ inline Sixteen<T> load_sixteen(const T *p, int n)
{
    constexpr int V = kVec<T>;
    Sixteen<T> s;
#pragma unroll
    for (int i = 0; i < 16 / V; ++i) s.p[i] = load_pack<T, V>(p + i * V, n - i * V);
    return s;
}
template <typename T>
__device__ inline void to_floats(const Sixteen<T> &s, float (&v)[16])
{
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = (float)s.p[i / kVec<T>][i % kVec<T>];
}

__device__ inline void count_values(uint64_t *status, uint32_t n)
{
    if (status && n) atomicAdd(reinterpret_cast<unsigned long long *>(status + CO3_STAT_NONFINITE), (unsigned long long)n);
}

// A workgroup takes a block of 128 x 128: eight threads have a row's columns, sixteen each, of every 32nd row.
template <typename T>
__global__ __launch_bounds__(256) void k_quantize8(co3_quantize8_args a, uint32_t first)
{
    __shared__ float most[4];
    const co3_blocks8 &o = a.out;
    const uint32_t block = first + blockIdx.x, col = blockIdx.y * kBlockCols + threadIdx.x % 8 * 16;
    const uint64_t row = (uint64_t)block * 128 + threadIdx.x / 8;
    const T *x = static_cast<const T *>(a.x) + blockIdx.z * a.x_batch_stride + col;
    const int n = (int)o.cols - (int)col;
    Sixteen<T> s[4];
    float m = 0.f;
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = load_sixteen<T>(x + (row + 32 * i) * a.x_stride, row + 32 * i < o.rows ? n : 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[16];
        to_floats(s[i], v);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            m = fmaxf(m, finite_size(v[k]));
            odd += fabsf(v[k]) < INFINITY ? 0u : 1u;
        }
    }
#pragma unroll
    for (int k = 32; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
    if (threadIdx.x % 64 == 0) most[threadIdx.x / 64] = m;
    __syncthreads();
    m = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
    const uint32_t byte = scale_byte(m);
    if (threadIdx.x == 0) o.scales[((uint64_t)blockIdx.z * block_columns(o) + blockIdx.y) * o.scale_ld + block] = (uint8_t)byte;
    count_values(a.status, odd);
    if (n <= 0) return;   // behind the last sixteen
    const float inverse = power_of(254 - byte);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (row + 32 * i >= o.rows) break;
        float v[16];
        to_floats(s[i], v);
        *reinterpret_cast<uint4 *>(o.values + blockIdx.z * o.batch_stride + (row + 32 * i) * o.ld + col) = bytes_of(v, inverse, odd != 0);
    }
}

// Blocks of one row: eight threads a block, 32 rows a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void k_quantize8_rows(co3_quantize8_args a, uint32_t first)
{
    const co3_blocks8 &o = a.out;
    const uint32_t col = blockIdx.y * kBlockCols + threadIdx.x % 8 * 16;
    const uint64_t row = (uint64_t)(first + blockIdx.x) * 32 + threadIdx.x / 8;
    if (row >= o.rows) return;   // all eight threads of the row
    const int n = (int)o.cols - (int)col;
    float v[16];
    to_floats(load_sixteen<T>(static_cast<const T *>(a.x) + blockIdx.z * a.x_batch_stride + row * a.x_stride + col, n), v);
    float m = 0.f;
    uint32_t odd = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        m = fmaxf(m, finite_size(v[k]));
        odd += fabsf(v[k]) < INFINITY ? 0u : 1u;
    }
#pragma unroll
    for (int k = 4; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
    const uint32_t byte = scale_byte(m);
    if (threadIdx.x % 8 == 0) o.scales[((uint64_t)blockIdx.z * block_columns(o) + blockIdx.y) * o.scale_ld + row] = (uint8_t)byte;
    count_values(a.status, odd);
    if (n <= 0) return;
    *reinterpret_cast<uint4 *>(o.values + blockIdx.z * o.batch_stride + row * o.ld + col) = bytes_of(v, power_of(254 - byte), odd != 0);
}

// A thread takes sixteen values, rows one behind the other in a workgroup's share.
template <typename T>
__global__ __launch_bounds__(256) void k_dequantize8(co3_dequantize8_args a, uint32_t first)
{
    const co3_blocks8 &x = a.x;
    constexpr float kMost = sizeof(T) == 4 ? 3.4028234663852886e38f : __is_same(T, __bf16) ? 3.3895313892515355e38f : 65504.f;
    const uint32_t col = blockIdx.y * kBlockCols + threadIdx.x % 8 * 16;
    const int n = (int)x.cols - (int)col;
    if (n <= 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t row = (uint64_t)(first + blockIdx.x) * 128 + 32 * i + threadIdx.x / 8;
        if (row >= x.rows) break;
        const uint64_t br = x.block_rows == 1 ? row : row / 128;
        const float scale = power_of(x.scales[((uint64_t)blockIdx.z * block_columns(x) + blockIdx.y) * x.scale_ld + br]);
        const uint4 w = *reinterpret_cast<const uint4 *>(x.values + blockIdx.z * x.batch_stride + row * x.ld + col);
        float v[16];
        numbers_of(w.x, v);
        numbers_of(w.y, v + 4);
        numbers_of(w.z, v + 8);
        numbers_of(w.w, v + 12);
        T *out = static_cast<T *>(a.out) + blockIdx.z * a.out_batch_stride + row * a.out_stride + col;
        constexpr int V = kVec<T>;
#pragma unroll
        for (int q = 0; q < 16 / V; ++q) {
            typename Pack<T, V>::V p;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                float f = v[q * V + k] * scale;
                f = f > kMost ? kMost : f < -kMost ? -kMost : f;   // NaN stays
                p[k] = (T)f;
            }
            store_pack<T, V>(out + q * V, n - q * V, p);
        }
    }
}

// A launch of HIP has fewer than 2^32 threads: `rows` workgroups of 256 for every column of blocks and matrix, in as many launches as it takes.
template <typename F>
static void launches(uint64_t rows, uint32_t columns, uint32_t batch, F &&launch)
{
    for (uint32_t m = 0; m < batch;) {
        const uint64_t most = ((1ull << 32) - 1) / 256 / columns;   // columns <= 2^13
        const uint32_t matrices = (uint32_t)(rows * (batch - m) <= most ? batch - m : most / rows ? most / rows : 1);
        for (uint64_t r = 0; r < rows; r += most) launch((uint32_t)r, dim3((uint32_t)(rows - r < most ? rows - r : most), columns, matrices), m);
        m += matrices;
    }
}

template <typename T>
static void quantize_of(const co3_quantize8_args &a, hipStream_t s)
{
    const bool single = a.out.block_rows == 1;
    launches(single ? (a.out.rows + 31) / 32 : (a.out.rows + 127) / 128, block_columns(a.out), a.out.batch, [&](uint32_t first, dim3 grid, uint32_t m) {
        co3_quantize8_args part = a;
        part.x = static_cast<const T *>(a.x) + m * a.x_batch_stride;
        part.out.values += m * a.out.batch_stride;
        part.out.scales += (uint64_t)m * block_columns(a.out) * a.out.scale_ld;
        if (single) k_quantize8_rows<T><<<grid, dim3(256), 0, s>>>(part, first);
        else k_quantize8<T><<<grid, dim3(256), 0, s>>>(part, first);
    });
}

template <typename T>
static void dequantize_of(const co3_dequantize8_args &a, hipStream_t s)
{
    launches((a.x.rows + 127) / 128, block_columns(a.x), a.x.batch, [&](uint32_t first, dim3 grid, uint32_t m) {
        co3_dequantize8_args part = a;
        part.out = static_cast<T *>(a.out) + m * a.out_batch_stride;
        part.x.values += m * a.x.batch_stride;
        part.x.scales += (uint64_t)m * block_columns(a.x) * a.x.scale_ld;
        k_dequantize8<T><<<grid, dim3(256), 0, s>>>(part, first);
    });
}

hipError_t launch_quantize8(const co3_quantize8_args &a, hipStream_t s)
{
    ProfScope prof(K_QUANTIZE8, s);
    if (a.type == CO3_F32) quantize_of<float>(a, s);
    else if (a.type == CO3_BF16) quantize_of<__bf16>(a, s);
    else quantize_of<_Float16>(a, s);
    return hipGetLastError();
}

hipError_t launch_dequantize8(const co3_dequantize8_args &a, hipStream_t s)
{
    ProfScope prof(K_DEQUANTIZE8, s);
    if (a.type == CO3_F32) dequantize_of<float>(a, s);
    else if (a.type == CO3_BF16) dequantize_of<__bf16>(a, s);
    else dequantize_of<_Float16>(a, s);
    return hipGetLastError();
}

}  // namespace co3
