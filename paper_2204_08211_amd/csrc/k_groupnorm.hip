// Group norm with an activation, channels last: forward pass, backward pass, the weight's gradients per user.
//
// Forward:   mean, var over a sample's pixels and a group's channels, rstd = 1 / sqrt(var + eps), z = (x - mean) rstd w + b, y = act(z)
// Backward:  xh = (x - mean) rstd,  z = xh w + b,  dz = dy act'(z).  Of every sample and channel
//            S1 = sum over the pixels of dz,  S2 = sum of dz xh;  over a group's channels m1 = mean(w S1), m2 = mean(w S2):
//            dx = rstd (dz w - m1 - xh m2),  dweight[u] = sum over the user's samples of S2,  dbias[u] = of S1
// so one pass over the data gives all sums, and a second one dx.
//
// Two ways.  Where a workgroup can hold a sample's pixels of some whole groups (128 bytes of a pixel or more) in registers, it reads them once
// and all is one launch.  Beyond that the sums of slices of pixels go through the workspace, and x (and dy) are read twice.
// All sums are formed in a fixed order.
#include <type_traits>

#include "blocks8.h"
#include "co3_internal.h"
#include "tensor_types.h"

namespace co3 {

struct Strip { uint32_t groups, blocks, packs; };   // groups of a workgroup, workgroups of a sample, packs of a pixel

template <typename T> struct Held { typename Pack<T, kVec<T>>::V v; };

__device__ inline float sigmoid(float z)
{
    // 1 / (1 + 2^(-z / ln 2)): exp2 and the reciprocal are good to a unit in the last place; 0 and 1 at the ends
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504088896340736f));
}
template <int ACT>
__device__ inline float activated(float z) { return ACT == CO3_ACT_RELU ? (z > 0.f ? z : z != z ? z : 0.f) : ACT == CO3_ACT_SILU ? z * sigmoid(z) : z; }
template <int ACT>
__device__ inline float slope(float z)
{
    if (ACT == CO3_ACT_RELU) return z > 0.f ? 1.f : 0.f;
    if (ACT != CO3_ACT_SILU) return 1.f;
    const float p = sigmoid(z);
    return p * (1.f + z * (1.f - p));
}

// V values of x from channel c of a row on: of `type`, or in 8 bits with the scale of their block.
template <typename T, bool KEPT> struct Input;
template <typename T> struct Input<T, false> {
    static constexpr int V = kVec<T>;
    typename Pack<T, V>::V p;
    __device__ inline void load(const co3_groupnorm_backward_args &a, uint64_t row, uint32_t c, int n)
    {
        p = load_pack<T, V>(static_cast<const T *>(a.x) + row * a.x_stride + c, n);
    }
    __device__ inline float get(int i) const { return (float)p[i]; }
    __device__ inline void pin() { asm volatile("" : "+v"(p)); }
};
template <typename T> struct Input<T, true> {
    static constexpr int V = kVec<T>;
    uint32_t words[V / 4];
    float low, high;      // scales: of the first values, of those from `turn` on
    int turn;
    __device__ inline void load(const co3_groupnorm_backward_args &a, uint64_t row, uint32_t c, int n)
    {
        const co3_blocks8 &x = a.x8;
        const uint32_t matrix = x.batch > 1 ? (uint32_t)(row / x.rows) : 0u;
        const uint64_t r = row - matrix * x.rows;
        const uint8_t *v = x.values + matrix * x.batch_stride + r * x.ld + c;
#pragma unroll
        for (int q = 0; q < V / 4; ++q) words[q] = 0;
        if (n >= V) {
            typedef uint32_t word __attribute__((aligned(1)));
#pragma unroll
            for (int q = 0; q < V / 4; ++q) words[q] = reinterpret_cast<const word *>(v)[q];
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < n) words[i / 4] |= (uint32_t)v[i] << (i % 4 * 8);
        }
        low = high = 0.f;
        if (n <= 0) return;
        const uint64_t br = x.block_rows == 1 ? r : r / 128;
        const uint32_t last = c + (n < V ? n : V) - 1;
        const uint8_t *s = x.scales + (uint64_t)matrix * block_columns(x) * x.scale_ld + br;
        low = power_of(s[(uint64_t)(c / kBlockCols) * x.scale_ld]);
        high = last / kBlockCols == c / kBlockCols ? low : power_of(s[(uint64_t)(last / kBlockCols) * x.scale_ld]);
        turn = (int)(kBlockCols - c % kBlockCols);
    }
    __device__ inline float get(int i) const
    {
        float v[4];
        numbers_of(words[i / 4], v);
        return v[i % 4] * (i < turn ? low : high);
    }
    __device__ inline void pin() { }
};

// red[rows][width] of a workgroup's threads -> red[q][c], q < rows left, which the return value is: sums over rows q, q + left, ...
template <int WG>
__device__ inline uint32_t fold_rows(float *red, uint32_t rows, uint32_t width)
{
    __syncthreads();
    uint32_t left = WG / width;
    left = left < 1 ? 1 : left < rows ? left : rows;
    if (left < rows) {
        for (uint32_t k = threadIdx.x; k < left * width; k += WG) {
            const uint32_t c = k % width, q = k / width;
            float s = red[q * width + c];
            for (uint32_t r = q + left; r < rows; r += left) s += red[r * width + c];
            red[q * width + c] = s;   // nobody else reads it
        }
        __syncthreads();
    }
    return left;
}

// out[g] = sum over q < rows and the group's channels of weight red[q][c]; weight may be NULL.
template <int WG>
__device__ inline void fold_groups(const float *red, uint32_t rows, uint32_t width, uint32_t groups, uint32_t per, const float *weight, float *out)
{
    for (uint32_t g = threadIdx.x / 64; g < groups; g += WG / 64) {
        float s = 0.f;
        for (uint32_t k = threadIdx.x % 64; k < rows * per; k += 64) {
            const uint32_t c = g * per + k % per;
            const float v = red[k / per * width + c];
            s += weight ? v * weight[c] : v;
        }
#pragma unroll
        for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
        if (threadIdx.x % 64 == 0) out[g] = s;
    }
    __syncthreads();
}

// ---- in one launch ------------------------------------------------------------------------------------------

template <typename T, int ACT, int WG, int CH>
__global__ __launch_bounds__(WG) void k_groupnorm(co3_groupnorm_args a, Strip strip, uint64_t first)
{
    constexpr int V = kVec<T>;
    extern __shared__ float red[];   // [rows][packs V], then the groups' sums
    const uint64_t sample = first + blockIdx.x;
    const uint32_t per = a.channels / a.groups, g0 = blockIdx.y * strip.groups, c0 = g0 * per;
    const uint32_t groups = a.groups - g0 < strip.groups ? a.groups - g0 : strip.groups, cn = groups * per;
    const uint32_t rows = WG / strip.packs, width = strip.packs * V, col = threadIdx.x % strip.packs, row = threadIdx.x / strip.packs, j = col * V;
    float *sums = red + rows * width;
    const int n = row < rows ? (int)cn - (int)j : 0;
    const uint32_t pixels = (uint32_t)a.pixels;
    const T *x = static_cast<const T *>(a.x) + sample * a.pixels * a.x_stride + c0 + j;
    typename Pack<T, V>::V p[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) p[i] = load_pack<T, V>(x + (uint64_t)(row + i * rows) * a.x_stride, row + i * rows < pixels ? n : 0);
    float s[V];
    const auto share = [&](float *out) {
        if (row < rows) {
#pragma unroll
            for (int k = 0; k < V; ++k) red[row * width + j + k] = s[k];
        }
        const uint32_t left = fold_rows<WG>(red, rows, width);
        fold_groups<WG>(red, left, width, groups, per, nullptr, out);
    };
#pragma unroll
    for (int k = 0; k < V; ++k) {
        s[k] = 0.f;
#pragma unroll
        for (int i = 0; i < CH; ++i) s[k] += (float)p[i][k];
    }
    share(sums);
    const float scale = 1.f / ((float)pixels * (float)per);
    float mean[V];
#pragma unroll
    for (int k = 0; k < V; ++k) mean[k] = k < n ? sums[(j + k) / per] * scale : 0.f;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        s[k] = 0.f;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const float d = (float)p[i][k] - mean[k];
            s[k] += row + i * rows < pixels && k < n ? d * d : 0.f;
        }
    }
    share(sums + groups);
    if (threadIdx.x < groups) {
        const uint64_t at = sample * a.groups + g0 + threadIdx.x;
        if (a.mean) a.mean[at] = sums[threadIdx.x] * scale;
        if (a.rstd) a.rstd[at] = 1.f / sqrtf(sums[groups + threadIdx.x] * scale + a.eps);
    }
    if (n <= 0) return;
    float f[V], b[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const bool in = k < n;
        const float rstd = in ? 1.f / sqrtf(sums[groups + (j + k) / per] * scale + a.eps) : 0.f;
        f[k] = in && a.weight ? rstd * a.weight[c0 + j + k] : rstd;
        b[k] = in && a.bias ? a.bias[c0 + j + k] : 0.f;
    }
    T *y = static_cast<T *>(a.y) + sample * a.pixels * a.y_stride + c0 + j;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        if (row + i * rows >= pixels) break;
        typename Pack<T, V>::V o;
#pragma unroll
        for (int k = 0; k < V; ++k) o[k] = (T)activated<ACT>(((float)p[i][k] - mean[k]) * f[k] + b[k]);
        store_pack<T, V>(y + (uint64_t)(row + i * rows) * a.y_stride, n, o);
    }
}

// A thread's channels in the backward pass.
template <int V>
struct Channels {
    float mean[V], rstd[V], w[V], b[V];
    __device__ inline void load(const co3_groupnorm_backward_args &a, uint64_t sample, uint32_t c, int n)
    {
        const uint32_t per = a.channels / a.groups;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const bool in = k < n;
            const uint64_t g = sample * a.groups + (c + k) / per;
            mean[k] = in ? a.mean[g] : 0.f;
            rstd[k] = in ? a.rstd[g] : 0.f;
            w[k] = in && a.weight ? a.weight[c + k] : 1.f;
            b[k] = in && a.bias ? a.bias[c + k] : 0.f;
        }
    }
    __device__ inline float xh(int k, float x) const { return (x - mean[k]) * rstd[k]; }
    template <int ACT>
    __device__ inline float dz(int k, float xh, float dy) const { return ACT == CO3_ACT_NONE ? dy : ACT == CO3_ACT_RELU ? (xh * w[k] + b[k] > 0.f ? dy : 0.f) : dy * slope<ACT>(xh * w[k] + b[k]); }
};

template <typename T, bool KEPT, int ACT, int WG, int CH>
__global__ __launch_bounds__(WG) void k_groupnorm_backward(co3_groupnorm_backward_args a, Strip strip, uint64_t first, float *partial)
{
    constexpr int V = kVec<T>;
    extern __shared__ float red[];
    const uint64_t sample = first + blockIdx.x;
    const uint32_t per = a.channels / a.groups, g0 = blockIdx.y * strip.groups, c0 = g0 * per;
    const uint32_t groups = a.groups - g0 < strip.groups ? a.groups - g0 : strip.groups, cn = groups * per;
    const uint32_t rows = WG / strip.packs, width = strip.packs * V, col = threadIdx.x % strip.packs, row = threadIdx.x / strip.packs, j = col * V;
    float *sums = red + rows * width;
    const int n = row < rows ? (int)cn - (int)j : 0;
    const uint32_t pixels = (uint32_t)a.pixels;
    const uint64_t r0 = sample * a.pixels;
    Input<T, KEPT> x[CH];
    typename Pack<T, V>::V d[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const uint32_t r = row + i * rows;
        const bool in = r < pixels;
        x[i].load(a, r0 + (in ? r : 0), c0 + j, in ? n : 0);
        d[i] = load_pack<T, V>(static_cast<const T *>(a.dy) + (r0 + r) * a.dy_stride + c0 + j, in ? n : 0);
    }
    Channels<V> ch;
    ch.load(a, sample, c0 + j, n);
    float s1[V], s2[V];
#pragma unroll
    for (int k = 0; k < V; ++k) s1[k] = s2[k] = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float xh = ch.xh(k, x[i].get(k)), dz = row + i * rows < pixels && k < n ? ch.template dz<ACT>(k, xh, (float)d[i][k]) : 0.f;
            s1[k] += dz;
            s2[k] += dz * (row + i * rows < pixels ? xh : 0.f);
        }
    const auto share = [&](const float (&s)[V], float *out, uint32_t which) {
        if (row < rows) {
#pragma unroll
            for (int k = 0; k < V; ++k) red[row * width + j + k] = s[k];
        }
        const uint32_t left = fold_rows<WG>(red, rows, width);
        if (partial) {
            for (uint32_t c = threadIdx.x; c < cn; c += WG) {
                float t = red[c];
                for (uint32_t q = 1; q < left; ++q) t += red[q * width + c];
                partial[(sample * 2 + which) * a.channels + c0 + c] = t;
            }
        }
        fold_groups<WG>(red, left, width, groups, per, a.weight ? a.weight + c0 : nullptr, out);
    };
    share(s1, sums, 0);
    share(s2, sums + groups, 1);
    if (n <= 0) return;
    const float scale = 1.f / ((float)pixels * (float)per);
    T *dx = static_cast<T *>(a.dx) + c0 + j;
    float m1[V], m2[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        m1[k] = k < n ? sums[(j + k) / per] * scale : 0.f;
        m2[k] = k < n ? sums[groups + (j + k) / per] * scale : 0.f;
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        if (row + i * rows >= pixels) break;
        typename Pack<T, V>::V o;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float xh = ch.xh(k, x[i].get(k)), dz = ch.template dz<ACT>(k, xh, (float)d[i][k]);
            o[k] = (T)(ch.rstd[k] * (dz * ch.w[k] - m1[k] - xh * m2[k]));
        }
        store_pack<T, V>(dx + (r0 + row + (uint64_t)i * rows) * a.dx_stride, n, o);
    }
}

// ---- by slices of pixels ------------------------------------------------------------------------------------

// Workgroups of 256 threads: `packs` of them next to each other in a pixel, so many columns of these, slices of the pixels.
struct Slices { uint32_t packs, columns, slices; };

__device__ inline uint32_t slice_begin(uint32_t pixels, uint32_t slices, uint32_t i) { return (uint32_t)((uint64_t)pixels * i / slices); }

// Sums of x and of its squares, in fp64: no mean harms the variance, and no finite fp32 input overflows.
template <typename T>
__global__ __launch_bounds__(256) void k_groupnorm_sums(co3_groupnorm_args a, Slices cut, uint64_t first, double *partial)
{
    constexpr int V = kVec<T>;
    __shared__ double red[256 * V];
    const uint64_t sample = first + blockIdx.z;
    const uint32_t rows = 256 / cut.packs, col = threadIdx.x % cut.packs, row = threadIdx.x / cut.packs, c = (blockIdx.y * cut.packs + col) * V, width = cut.packs * V;
    const int n = row < rows ? (int)a.channels - (int)c : 0;
    const uint32_t end = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x + 1);
    const T *x = static_cast<const T *>(a.x) + sample * a.pixels * a.x_stride + c;
    double s[V], q[V];
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = q[k] = 0.0;
    if (n > 0) {
#pragma unroll 4
        for (uint32_t r = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x) + row; r < end; r += rows) {
            const auto p = load_pack<T, V>(x + r * a.x_stride, n);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const double v = (double)(float)p[k];
                s[k] += v;
                q[k] = __builtin_fma(v, v, q[k]);
            }
        }
    }
    double *out = partial + ((sample * cut.slices + blockIdx.x) * 2) * a.channels;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
        if (row < rows) {
#pragma unroll
            for (int k = 0; k < V; ++k) red[row * width + col * V + k] = which ? q[k] : s[k];
        }
        __syncthreads();
        for (uint32_t k = threadIdx.x; k < width; k += 256) {
            const uint32_t to = blockIdx.y * width + k;
            if (to >= a.channels) continue;
            double t = red[k];
            for (uint32_t r = 1; r < rows; ++r) t += red[r * width + k];
            out[(uint64_t)which * a.channels + to] = t;
        }
    }
}

// mean and rstd of a group, a wavefront each.
__global__ __launch_bounds__(256) void k_groupnorm_stats(co3_groupnorm_args a, uint32_t slices, uint64_t first, const double *partial, float *mean, float *rstd)
{
    const uint64_t k = first + (uint64_t)blockIdx.x * 4 + threadIdx.x / 64;
    if (k >= a.samples * a.groups) return;
    const uint64_t sample = k / a.groups;
    const uint32_t per = a.channels / a.groups, c0 = (uint32_t)(k % a.groups) * per;
    double s = 0.0, q = 0.0;
    for (uint32_t e = threadIdx.x % 64; e < slices * per; e += 64) {
        const double *p = partial + (sample * slices + e / per) * 2 * a.channels + c0 + e % per;
        s += p[0];
        q += p[a.channels];
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        s += __shfl_xor(s, o);
        q += __shfl_xor(q, o);
    }
    if (threadIdx.x % 64) return;
    const double n = 1.0 / ((double)a.pixels * per), m = s * n, var = q * n - m * m;
    mean[k] = (float)m;
    rstd[k] = (float)(1.0 / sqrt((var > 0.0 ? var : var != var ? var : 0.0) + (double)a.eps));
}

template <typename T, int ACT>
__global__ __launch_bounds__(256) void k_groupnorm_apply(co3_groupnorm_args a, Slices cut, uint64_t first, const float *mean, const float *rstd)
{
    constexpr int V = kVec<T>;
    const uint64_t sample = first + blockIdx.z;
    const uint32_t rows = 256 / cut.packs, col = threadIdx.x % cut.packs, row = threadIdx.x / cut.packs, c = (blockIdx.y * cut.packs + col) * V;
    const int n = row < rows ? (int)a.channels - (int)c : 0;
    if (n <= 0) return;
    const uint32_t end = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x + 1), per = a.channels / a.groups;
    float m[V], f[V], b[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const bool in = k < n;
        const uint64_t g = sample * a.groups + (c + k) / per;
        m[k] = in ? mean[g] : 0.f;
        f[k] = in ? (a.weight ? rstd[g] * a.weight[c + k] : rstd[g]) : 0.f;
        b[k] = in && a.bias ? a.bias[c + k] : 0.f;
    }
    const T *x = static_cast<const T *>(a.x) + sample * a.pixels * a.x_stride + c;
    T *y = static_cast<T *>(a.y) + sample * a.pixels * a.y_stride + c;
#pragma unroll 4
    for (uint32_t r = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x) + row; r < end; r += rows) {
        const auto p = load_pack<T, V>(x + r * a.x_stride, n);
        typename Pack<T, V>::V o;
#pragma unroll
        for (int k = 0; k < V; ++k) o[k] = (T)activated<ACT>(((float)p[k] - m[k]) * f[k] + b[k]);
        store_pack<T, V>(y + r * a.y_stride, n, o);
    }
}

// S1 and S2 of a slice of a sample's pixels, fp32: at most 512 terms in an accumulator.
template <typename T, bool KEPT, int ACT>
__global__ __launch_bounds__(256) void k_groupnorm_backward_sums(co3_groupnorm_backward_args a, Slices cut, uint64_t first, float *partial)
{
    constexpr int V = kVec<T>;
    __shared__ float red[256 * V];
    const uint64_t sample = first + blockIdx.z;
    const uint32_t rows = 256 / cut.packs, col = threadIdx.x % cut.packs, row = threadIdx.x / cut.packs, c = (blockIdx.y * cut.packs + col) * V, width = cut.packs * V;
    const int n = row < rows ? (int)a.channels - (int)c : 0;
    const uint32_t end = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x + 1);
    const uint64_t r0 = sample * a.pixels;
    float s1[V], s2[V];
#pragma unroll
    for (int k = 0; k < V; ++k) s1[k] = s2[k] = 0.f;
    if (n > 0) {
        Channels<V> ch;
        ch.load(a, sample, c, n);
#pragma unroll 2
        for (uint32_t r = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x) + row; r < end; r += rows) {
            Input<T, KEPT> x;
            x.load(a, r0 + r, c, n);
            const auto d = load_pack<T, V>(static_cast<const T *>(a.dy) + (r0 + r) * a.dy_stride + c, n);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float xh = ch.xh(k, x.get(k)), dz = ch.template dz<ACT>(k, xh, (float)d[k]);
                s1[k] += dz;
                s2[k] += dz * xh;
            }
        }
    }
    float *out = partial + ((sample * cut.slices + blockIdx.x) * 2) * a.channels;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
        if (row < rows) {
#pragma unroll
            for (int k = 0; k < V; ++k) red[row * width + col * V + k] = which ? s2[k] : s1[k];
        }
        const uint32_t left = fold_rows<256>(red, rows, width);
        for (uint32_t k = threadIdx.x; k < width; k += 256) {
            const uint32_t to = blockIdx.y * width + k;
            if (to >= a.channels) continue;
            float t = red[k];
            for (uint32_t q = 1; q < left; ++q) t += red[q * width + k];
            out[(uint64_t)which * a.channels + to] = t;
        }
    }
}

// m1 and m2 of a group, a wavefront each.
__global__ __launch_bounds__(256) void k_groupnorm_means(co3_groupnorm_backward_args a, uint32_t slices, uint64_t first, const float *partial, float *means)
{
    const uint64_t k = first + (uint64_t)blockIdx.x * 4 + threadIdx.x / 64;
    if (k >= a.U * a.samples_per_user * a.groups) return;
    const uint64_t sample = k / a.groups;
    const uint32_t per = a.channels / a.groups, c0 = (uint32_t)(k % a.groups) * per;
    double s1 = 0.0, s2 = 0.0;
    for (uint32_t e = threadIdx.x % 64; e < slices * per; e += 64) {
        const uint32_t c = c0 + e % per;
        const float *p = partial + (sample * slices + e / per) * 2 * a.channels + c;
        const double w = a.weight ? a.weight[c] : 1.f;
        s1 += w * p[0];
        s2 += w * p[a.channels];
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        s1 += __shfl_xor(s1, o);
        s2 += __shfl_xor(s2, o);
    }
    if (threadIdx.x % 64) return;
    const double n = 1.0 / ((double)a.pixels * per);
    means[2 * k] = (float)(s1 * n);
    means[2 * k + 1] = (float)(s2 * n);
}

template <typename T, bool KEPT, int ACT>
__global__ __launch_bounds__(256) void k_groupnorm_backward_apply(co3_groupnorm_backward_args a, Slices cut, uint64_t first, const float *means)
{
    constexpr int V = kVec<T>;
    const uint64_t sample = first + blockIdx.z;
    const uint32_t rows = 256 / cut.packs, col = threadIdx.x % cut.packs, row = threadIdx.x / cut.packs, c = (blockIdx.y * cut.packs + col) * V;
    const int n = row < rows ? (int)a.channels - (int)c : 0;
    if (n <= 0) return;
    const uint32_t end = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x + 1), per = a.channels / a.groups;
    const uint64_t r0 = sample * a.pixels;
    Channels<V> ch;
    ch.load(a, sample, c, n);
    float m1[V], m2[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const uint64_t g = sample * a.groups + (c + k) / per;
        m1[k] = k < n ? means[2 * g] : 0.f;
        m2[k] = k < n ? means[2 * g + 1] : 0.f;
    }
    T *dx = static_cast<T *>(a.dx) + c;
#pragma unroll 2
    for (uint32_t r = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x) + row; r < end; r += rows) {
        Input<T, KEPT> x;
        x.load(a, r0 + r, c, n);
        const auto d = load_pack<T, V>(static_cast<const T *>(a.dy) + (r0 + r) * a.dy_stride + c, n);
        typename Pack<T, V>::V o;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float xh = ch.xh(k, x.get(k)), dz = ch.template dz<ACT>(k, xh, (float)d[k]);
            o[k] = (T)(ch.rstd[k] * (dz * ch.w[k] - m1[k] - xh * m2[k]));
        }
        store_pack<T, V>(dx + (r0 + r) * a.dx_stride, n, o);
    }
}

// The users' gradients of the sums of `parts` (samples, or slices of them) each, 64 channels of either a workgroup, a wavefront every
// sixteenth part.  In fp64, since there may be thousands.
__global__ __launch_bounds__(1024) void k_groupnorm_grad(co3_groupnorm_backward_args a, uint64_t parts, uint32_t first, const float *partial)
{
    __shared__ double part[16][64];
    const uint32_t u = first + blockIdx.y, lane = threadIdx.x & 63u, w = threadIdx.x >> 6;
    const uint64_t c = (uint64_t)blockIdx.x * 64 + lane, channels = a.channels;   // dbias's columns, then dweight's
    double s = 0.0;
    if (c < 2 * channels) {
        const float *p = partial + u * parts * 2 * channels + c;
#pragma unroll 8
        for (uint64_t k = w; k < parts; k += 16) s += (double)p[k * 2 * channels];
    }
    part[w][lane] = s;
    __syncthreads();
    if (w || c >= 2 * channels) return;
    s = 0.0;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += part[k][lane];
    float *out = c < channels ? a.dbias : a.dweight;
    if (!out) return;
    out += u * a.grad_stride + (c < channels ? c : c - channels);
    *out = (float)(a.accumulate ? (double)*out + s : s);
}

// ---- launches -----------------------------------------------------------------------------------------------

static inline uint32_t elements_of_pack(int32_t type) { return type == CO3_F32 ? 4 : 8; }

// One launch: groups of 128 bytes of a pixel or more to a workgroup, of as few threads as hold them in `most` packs each.  threads = 0: too large.
struct Whole { Strip strip; uint32_t threads, held; };
static Whole whole_of(uint64_t pixels, uint32_t channels, uint32_t groups, int32_t type, uint32_t most)
{
    const uint32_t V = elements_of_pack(type), per = channels / groups;
    Whole w = {};
    w.strip.groups = (8 * V + per - 1) / per;
    if (w.strip.groups > groups) w.strip.groups = groups;
    w.strip.blocks = (groups + w.strip.groups - 1) / w.strip.groups;
    w.strip.packs = (w.strip.groups * per + V - 1) / V;
    const uint32_t sizes[3] = {64, 256, 1024};
    for (int k = 0; k < 3; ++k) {
        const uint32_t rows = sizes[k] / w.strip.packs;
        if (!rows) continue;
        const uint64_t held = (pixels + rows - 1) / rows;
        if (held > (k == 2 ? most : 4)) continue;
        w.threads = sizes[k];
        w.held = held <= 1 ? 1 : held <= 2 ? 2 : held <= 4 ? 4 : 8;
        break;
    }
    return w;
}
static inline uint32_t whole_lds(const Whole &w, int32_t type)
{
    return (w.threads / w.strip.packs * w.strip.packs * elements_of_pack(type) + 2 * w.strip.groups) * sizeof(float);
}

static Slices slices_of(uint64_t samples, uint64_t pixels, uint32_t channels, int32_t type, uint64_t most_terms)
{
    Slices s;
    const uint32_t packs = (channels + elements_of_pack(type) - 1) / elements_of_pack(type);
    s.packs = packs < 32 ? packs : 32;
    s.columns = (packs + s.packs - 1) / s.packs;
    const uint32_t rows = 256 / s.packs;
    const uint64_t fill = (2048 + samples * s.columns - 1) / (samples * s.columns), room = (pixels + 8 * rows - 1) / (8 * rows);
    uint64_t n = fill < room ? fill : room;
    const uint64_t least = (pixels + rows * most_terms - 1) / (rows * most_terms);
    if (n < least) n = least;
    s.slices = (uint32_t)(n < 1 ? 1 : n);
    return s;
}

static inline size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }
constexpr uint32_t kHeldForward = 8, kHeldBackward = 4;
constexpr uint64_t kNoLimit = 1ull << 31, kMostTerms = 512;

size_t groupnorm_workspace_bytes(uint64_t samples, uint64_t pixels, uint32_t channels, uint32_t groups, int32_t type)
{
    if (samples == 0 || whole_of(pixels, channels, groups, type, kHeldForward).threads) return 0;
    const Slices c = slices_of(samples, pixels, channels, type, kNoLimit);
    return samples * c.slices * 2 * channels * sizeof(double) + 2 * up16(samples * groups * sizeof(float));
}

size_t groupnorm_backward_workspace_bytes(uint32_t U, uint64_t samples_per_user, uint64_t pixels, uint32_t channels, uint32_t groups, int32_t type)
{
    const uint64_t samples = U * samples_per_user;
    if (samples == 0) return 0;
    if (whole_of(pixels, channels, groups, type, kHeldBackward).threads) return samples * 2 * channels * sizeof(float);
    const Slices c = slices_of(samples, pixels, channels, type, kMostTerms);
    return up16(samples * c.slices * 2 * channels * sizeof(float)) + samples * groups * 2 * sizeof(float);
}

// A launch of HIP has fewer than 2^32 threads: `threads` for each of `count`, at most `at_once` of them in one.
template <typename F>
static void in_parts(uint64_t count, uint64_t threads, uint64_t at_once, F &&launch)
{
    const uint64_t room = ((1ull << 32) - 1) / threads, most = room < at_once ? room : at_once;
    for (uint64_t i = 0; i < count; i += most) launch(i, (uint32_t)(count - i < most ? count - i : most));
}

template <typename F>
static void with_activation(int32_t activation, F &&f)
{
    if (activation == CO3_ACT_RELU) f(std::integral_constant<int, CO3_ACT_RELU>());
    else if (activation == CO3_ACT_SILU) f(std::integral_constant<int, CO3_ACT_SILU>());
    else f(std::integral_constant<int, CO3_ACT_NONE>());
}

// f(threads, packs held) of the forms that there are.
template <int MOST, typename F>
static void with_form(const Whole &w, F &&f)
{
    const auto held = [&](auto threads) {
        if (w.held == 1) f(threads, std::integral_constant<int, 1>());
        else if (w.held == 2) f(threads, std::integral_constant<int, 2>());
        else if (w.held == 4) f(threads, std::integral_constant<int, 4>());
        else if constexpr (MOST >= 8 && decltype(threads)::value == 1024) f(threads, std::integral_constant<int, 8>());
    };
    if (w.threads == 64) held(std::integral_constant<int, 64>());
    else if (w.threads == 256) held(std::integral_constant<int, 256>());
    else held(std::integral_constant<int, 1024>());
}

template <typename T>
static void forward_of(const co3_groupnorm_args &a, hipStream_t s)
{
    const Whole w = whole_of(a.pixels, a.channels, a.groups, a.type, kHeldForward);
    if (w.threads) {
        ProfScope prof(K_GROUPNORM, s);
        with_activation(a.activation, [&](auto act) {
            with_form<kHeldForward>(w, [&](auto threads, auto held) {
                constexpr int WG = decltype(threads)::value;
                in_parts(a.samples, (uint64_t)WG * w.strip.blocks, ~0ull, [&](uint64_t first, uint32_t count) {
                    k_groupnorm<T, decltype(act)::value, WG, decltype(held)::value>
                        <<<dim3(count, w.strip.blocks), dim3(WG), whole_lds(w, a.type), s>>>(a, w.strip, first);
                });
            });
        });
        return;
    }
    const Slices c = slices_of(a.samples, a.pixels, a.channels, a.type, kNoLimit);
    double *partial = static_cast<double *>(a.workspace);
    float *own = reinterpret_cast<float *>(partial + a.samples * c.slices * 2 * a.channels);
    float *mean = a.mean ? a.mean : own, *rstd = a.rstd ? a.rstd : own + up16(a.samples * a.groups * sizeof(float)) / sizeof(float);
    {
        ProfScope prof(K_GROUPNORM_SUMS, s);
        in_parts(a.samples, (uint64_t)256 * c.slices * c.columns, 65535, [&](uint64_t first, uint32_t count) {
            k_groupnorm_sums<T><<<dim3(c.slices, c.columns, count), dim3(256), 0, s>>>(a, c, first, partial);
        });
        in_parts((a.samples * a.groups + 3) / 4, 256, ~0ull, [&](uint64_t first, uint32_t count) {
            k_groupnorm_stats<<<dim3(count), dim3(256), 0, s>>>(a, c.slices, first * 4, partial, mean, rstd);
        });
    }
    ProfScope prof(K_GROUPNORM, s);
    with_activation(a.activation, [&](auto act) {
        in_parts(a.samples, (uint64_t)256 * c.slices * c.columns, 65535, [&](uint64_t first, uint32_t count) {
            k_groupnorm_apply<T, decltype(act)::value><<<dim3(c.slices, c.columns, count), dim3(256), 0, s>>>(a, c, first, mean, rstd);
        });
    });
}

template <typename T, bool KEPT>
static void backward_of(const co3_groupnorm_backward_args &a, hipStream_t s)
{
    const uint64_t samples = a.U * a.samples_per_user;
    const Whole w = whole_of(a.pixels, a.channels, a.groups, a.type, kHeldBackward);
    float *partial = static_cast<float *>(a.workspace);
    const bool grads = a.dweight || a.dbias;
    uint64_t parts = a.samples_per_user;
    if (samples && w.threads) {
        ProfScope prof(K_GROUPNORM_BACKWARD, s);
        with_activation(a.activation, [&](auto act) {
            with_form<kHeldBackward>(w, [&](auto threads, auto held) {
                constexpr int WG = decltype(threads)::value;
                in_parts(samples, (uint64_t)WG * w.strip.blocks, ~0ull, [&](uint64_t first, uint32_t count) {
                    k_groupnorm_backward<T, KEPT, decltype(act)::value, WG, decltype(held)::value>
                        <<<dim3(count, w.strip.blocks), dim3(WG), whole_lds(w, a.type), s>>>(a, w.strip, first, grads ? partial : nullptr);
                });
            });
        });
    } else if (samples) {
        const Slices c = slices_of(samples, a.pixels, a.channels, a.type, kMostTerms);
        parts *= c.slices;
        float *means = partial + up16(samples * c.slices * 2 * a.channels * sizeof(float)) / sizeof(float);
        with_activation(a.activation, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            {
                ProfScope prof(K_GROUPNORM_SUMS, s);
                in_parts(samples, (uint64_t)256 * c.slices * c.columns, 65535, [&](uint64_t first, uint32_t count) {
                    k_groupnorm_backward_sums<T, KEPT, ACT><<<dim3(c.slices, c.columns, count), dim3(256), 0, s>>>(a, c, first, partial);
                });
                in_parts((samples * a.groups + 3) / 4, 256, ~0ull, [&](uint64_t first, uint32_t count) {
                    k_groupnorm_means<<<dim3(count), dim3(256), 0, s>>>(a, c.slices, first * 4, partial, means);
                });
            }
        });
        if (grads) {   // before dx, which may take x's place, is no matter: all sums are there
            ProfScope prof(K_GROUPNORM_GRAD, s);
            in_parts(a.U, (uint64_t)1024 * ((2 * a.channels + 63) / 64), 65535, [&](uint64_t first, uint32_t count) {
                k_groupnorm_grad<<<dim3((2 * a.channels + 63) / 64, count), dim3(1024), 0, s>>>(a, parts, (uint32_t)first, partial);
            });
        }
        ProfScope prof(K_GROUPNORM_BACKWARD, s);
        with_activation(a.activation, [&](auto act) {
            in_parts(samples, (uint64_t)256 * c.slices * c.columns, 65535, [&](uint64_t first, uint32_t count) {
                k_groupnorm_backward_apply<T, KEPT, decltype(act)::value><<<dim3(c.slices, c.columns, count), dim3(256), 0, s>>>(a, c, first, means);
            });
        });
        return;
    }
    if (!grads) return;
    ProfScope prof(K_GROUPNORM_GRAD, s);
    in_parts(a.U, (uint64_t)1024 * ((2 * a.channels + 63) / 64), 65535, [&](uint64_t first, uint32_t count) {
        k_groupnorm_grad<<<dim3((2 * a.channels + 63) / 64, count), dim3(1024), 0, s>>>(a, parts, (uint32_t)first, partial);
    });
}

hipError_t launch_groupnorm(const co3_groupnorm_args &a, hipStream_t s)
{
    if (a.type == CO3_F32) forward_of<float>(a, s);
    else if (a.type == CO3_BF16) forward_of<__bf16>(a, s);
    else forward_of<_Float16>(a, s);
    return hipGetLastError();
}

hipError_t launch_groupnorm_backward(const co3_groupnorm_backward_args &a, hipStream_t s)
{
    const auto go = [&](auto kept) {
        constexpr bool KEPT = decltype(kept)::value;
        if (a.type == CO3_F32) backward_of<float, KEPT>(a, s);
        else if (a.type == CO3_BF16) backward_of<__bf16, KEPT>(a, s);
        else backward_of<_Float16, KEPT>(a, s);
    };
    if (a.x) go(std::false_type());
    else go(std::true_type());
    return hipGetLastError();
}

}  // namespace co3
