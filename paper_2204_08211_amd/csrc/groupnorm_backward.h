// Group norm's backward pass, for the two files that instantiate it: k_groupnorm_backward.hip (x as it is) and k_groupnorm_backward8.hip (x
// kept in 8 bits).  The mathematics are at the head of k_groupnorm.hip.
#pragma once

#include "groupnorm.h"

namespace co3 {

// A sample's x: fetch() asks for a pack, numbers() makes fp32 of it, so that many are on their way at a time.  ONE: packs are whole and
// lie in one block.
template <typename T, bool KEPT, bool ONE> struct Source;
template <typename T, bool ONE> struct Source<T, false, ONE> {
    typedef typename Pack<T, kVec<T>>::V Raw;
    const T *x;
    uint64_t stride;
    __device__ inline Source(const co3_groupnorm_backward_args &a, uint64_t sample, uint32_t c)
        : x(static_cast<const T *>(a.x) + sample * a.pixels * a.x_stride + c), stride(a.x_stride) { }
    template <bool FULL>
    __device__ inline Raw fetch(uint32_t pixel, const Lane<kVec<T>, ONE> &lane, bool there) const { return load_lane<FULL>(x + pixel * stride, lane, there); }
    __device__ inline typename Pack<float, kVec<T>>::V numbers(const Raw &r) const
    {
        typename Pack<float, kVec<T>>::V p;
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) p[i] = (float)r[i];
        return p;
    }
};
template <typename T, bool ONE> struct Source<T, true, ONE> {
    static constexpr int V = kVec<T>;
    struct Raw { uint32_t words[V / 4], low, high; };
    const uint8_t *values, *low, *high;   // low, high: of the first channel's block, of the one that the last of V lies in
    uint32_t ld, row, shift;
    int turn;                             // channels of the first block
    __device__ inline Source(const co3_groupnorm_backward_args &a, uint64_t sample, uint32_t c)
    {
        const co3_blocks8 &x = a.x8;
        const uint32_t matrix = x.batch > 1 ? (uint32_t)sample / (uint32_t)a.samples_per_user : 0u;
        row = ((uint32_t)sample - (x.batch > 1 ? matrix * (uint32_t)a.samples_per_user : 0u)) * (uint32_t)a.pixels;
        values = x.values + matrix * x.batch_stride + c;
        const uint32_t block = c / kBlockCols, next = (c + V - 1) / kBlockCols, last = (x.cols - 1) / kBlockCols;
        low = x.scales + ((uint64_t)matrix * block_columns(x) + (block < last ? block : last)) * x.scale_ld;
        high = x.scales + ((uint64_t)matrix * block_columns(x) + (next < last ? next : last)) * x.scale_ld;
        ld = (uint32_t)x.ld;
        shift = x.block_rows == 1 ? 0 : 7;
        turn = (int)(kBlockCols - c % kBlockCols);
    }
    template <bool FULL>
    __device__ inline Raw fetch(uint32_t pixel, const Lane<V, ONE> &lane, bool there) const
    {
        const int n = there ? lane.n : 0;
        Raw p;
#pragma unroll
        for (int q = 0; q < V / 4; ++q) p.words[q] = 0;
        p.low = p.high = 127;
        if (n <= 0) return p;
        const uint32_t r = row + pixel;
        const uint8_t *v = values + (uint64_t)r * ld;
        if (FULL) {
            typedef uint32_t word __attribute__((aligned(1)));
#pragma unroll
            for (int q = 0; q < V / 4; ++q) p.words[q] = reinterpret_cast<const word *>(v)[q];
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < n) p.words[i / 4] |= (uint32_t)v[i] << (i % 4 * 8);
        }
        p.low = low[r >> shift];
        if (!ONE) p.high = high[r >> shift];
        return p;
    }
    __device__ inline typename Pack<float, V>::V numbers(const Raw &r) const
    {
        typename Pack<float, V>::V p;
        const float f = power_of(r.low), g = ONE ? f : power_of(r.high);
        float w[V];
#pragma unroll
        for (int q = 0; q < V / 4; ++q) numbers_of(r.words[q], w + 4 * q);
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] = w[i] * (ONE || i < turn ? f : g);
        return p;
    }
};

// ---- in one launch ------------------------------------------------------------------------------------------

// A thread's channels in the backward pass; ONE: of one group.
template <int V, bool ONE>
struct Channels {
    float mean[ONE ? 1 : V], rstd[ONE ? 1 : V], w[V], b[V];
    __device__ inline void load(const co3_groupnorm_backward_args &a, uint64_t sample, const Lane<V, ONE> &lane)
    {
        typename Pack<float, V>::V pw, pb;
#pragma unroll
        for (int k = 0; k < V; ++k) { pw[k] = 1.f; pb[k] = 0.f; }
#pragma unroll
        for (int k = 0; k < (ONE ? 1 : V); ++k) mean[k] = rstd[k] = 0.f;
        if (lane.n > 0) {
            for_groups(lane, 0, a.channels / a.groups, [&](int k, uint32_t g) {
                mean[k] = a.mean[sample * a.groups + g];
                rstd[k] = a.rstd[sample * a.groups + g];
            });
            if (a.weight) pw = load_pack<float, V>(a.weight + lane.base, ONE ? V : lane.n);
            if (a.bias) pb = load_pack<float, V>(a.bias + lane.base, ONE ? V : lane.n);
        }
#pragma unroll
        for (int k = 0; k < V; ++k) { w[k] = pw[k]; b[k] = pb[k]; }
    }
    __device__ inline float xh(int k, float x) const { return (x - mean[ONE ? 0 : k]) * rstd[ONE ? 0 : k]; }
    // rstd (dz w - m1 - xh m2), from rstd m1 and rstd m2
    __device__ inline float dx(int k, float xh, float dz, float m1, float m2) const
    {
        return __builtin_fmaf(dz * w[k], rstd[ONE ? 0 : k], -__builtin_fmaf(xh, m2, m1));
    }
};

template <typename T, bool KEPT, int ACT, int WG, int CH, bool ONE>
__global__ __launch_bounds__(WG, 4) void k_groupnorm_backward(co3_groupnorm_backward_args a, Strip strip, uint64_t first, float *partial)
{
    constexpr int V = kVec<T>;
    extern __shared__ float sums[];   // two of every group, then what the channels' sums take
    const uint64_t sample = first + blockIdx.x;
    const uint32_t per = a.channels / a.groups, g0 = blockIdx.y * strip.groups, c0 = g0 * per;
    const uint32_t groups = a.groups - g0 < strip.groups ? a.groups - g0 : strip.groups, cn = groups * per;
    const uint32_t rows = WG / strip.packs, width = strip.packs * V, row = threadIdx.x / strip.packs, pixels = (uint32_t)a.pixels;
    float *red = sums + 2 * strip.groups;
    const Lane<V, ONE> lane(c0, cn, threadIdx.x % strip.packs * V, true);
    const Source<T, KEPT, ONE> source(a, sample, lane.base);
    const T *dy = static_cast<const T *>(a.dy) + sample * a.pixels * a.dy_stride + lane.base;
    typename Source<T, KEPT, ONE>::Raw raw[CH];
    typename Pack<T, V>::V d[CH];
    with_rows<V, ONE>(a.channels, [&](auto full) {
        constexpr bool FULL = decltype(full)::value;
#pragma unroll
        for (int i = 0; i < CH; ++i) raw[i] = source.template fetch<FULL>(row + i * rows, lane, row + i * rows < pixels);
#pragma unroll
        for (int i = 0; i < CH; ++i) d[i] = load_lane<FULL>(dy + (row + i * rows) * a.dy_stride, lane, row + i * rows < pixels);
    });
    Channels<V, ONE> ch;
    ch.load(a, sample, lane);
    float s1[V], s2[V];
#pragma unroll
    for (int k = 0; k < V; ++k) s1[k] = s2[k] = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        if (row + i * rows >= pixels) continue;
        const auto x = source.numbers(raw[i]);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float xh = ch.xh(k, x[k]), dz = passed<ACT>((float)d[i][k], xh, ch.w[k], ch.b[k]);
            s1[k] += dz;
            s2[k] = __builtin_fmaf(dz, xh, s2[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (!lane.own(k)) s1[k] = s2[k] = 0.f;
    fold_channels<V, WG>(s1, s2, red, strip.packs);   // totals of S1, then of S2
    if (partial) {
        for (uint32_t c = threadIdx.x; c < cn; c += WG) {
            const uint32_t at = place_of<V>(c0, cn, c);
            partial[sample * 2 * a.channels + c0 + c] = red[at];
            partial[(sample * 2 + 1) * a.channels + c0 + c] = red[width + at];
        }
    }
    fold_groups<WG, V, float>(groups, per, c0, cn, [&](uint32_t at, uint32_t c, float &s, float &q) {
        const float w = a.weight ? a.weight[c0 + c] : 1.f;
        s += w * red[at];
        q += w * red[width + at];
    }, [&](uint32_t g, float s, float q) {
        sums[g] = s;
        sums[groups + g] = q;
    });
    if (lane.n <= 0) return;
    const float scale = 1.f / ((float)pixels * (float)per);
    T *dx = static_cast<T *>(a.dx) + sample * a.pixels * a.dx_stride + lane.base;
    float m1[ONE ? 1 : V] = {}, m2[ONE ? 1 : V] = {};
    for_groups(lane, c0, per, [&](int k, uint32_t g) {
        m1[k] = sums[g] * scale * ch.rstd[k];
        m2[k] = sums[groups + g] * scale * ch.rstd[k];
    });
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const uint32_t r = row + i * rows;
        if (r >= pixels) continue;
        const auto x = source.numbers(raw[i]);
        typename Pack<T, V>::V o;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float xh = ch.xh(k, x[k]), dz = passed<ACT>((float)d[i][k], xh, ch.w[k], ch.b[k]);
            o[k] = (T)ch.dx(k, xh, dz, m1[ONE ? 0 : k], m2[ONE ? 0 : k]);
        }
        store_lane<T, ONE>(dx + r * a.dx_stride, lane, o);
    }
}

// ---- by slices of pixels ------------------------------------------------------------------------------------

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

// S1 and S2 of a slice of a sample's pixels, fp32: at most 512 terms in an accumulator.
template <typename T, bool KEPT, int ACT, bool ONE>
__global__ __launch_bounds__(256) void k_groupnorm_backward_sums(co3_groupnorm_backward_args a, Slices cut, uint64_t first, float *partial)
{
    constexpr int V = kVec<T>;
    __shared__ float red[256 * V];
    const uint64_t sample = first + blockIdx.z;
    const uint32_t rows = 256 / cut.packs, col = threadIdx.x % cut.packs, row = threadIdx.x / cut.packs, width = cut.packs * V;
    const Lane<V, ONE> lane(0, a.channels, (blockIdx.y * cut.packs + col) * V, row < rows);
    const uint32_t end = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x + 1);
    float s1[V], s2[V];
#pragma unroll
    for (int k = 0; k < V; ++k) s1[k] = s2[k] = 0.f;
    if (lane.n > 0) {
        Channels<V, ONE> ch;
        ch.load(a, sample, lane);
        const Source<T, KEPT, ONE> source(a, sample, lane.base);
        const T *dy = static_cast<const T *>(a.dy) + sample * a.pixels * a.dy_stride + lane.base;
        with_rows<V, ONE>(a.channels, [&](auto full) {
            constexpr bool FULL = decltype(full)::value;
            for (uint32_t r = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x) + row; r < end; r += kAtOnce * rows) {
                typename Source<T, KEPT, ONE>::Raw raw[kAtOnce];
                typename Pack<T, V>::V d[kAtOnce];
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    raw[i] = source.template fetch<FULL>(r + i * rows, lane, r + i * rows < end);
                    d[i] = load_lane<FULL>(dy + (r + i * rows) * a.dy_stride, lane, r + i * rows < end);
                }
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    if (r + i * rows >= end) continue;
                    const auto x = source.numbers(raw[i]);
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        const float xh = ch.xh(k, x[k]), dz = passed<ACT>((float)d[i][k], xh, ch.w[k], ch.b[k]);
                        s1[k] += dz;
                        s2[k] = __builtin_fmaf(dz, xh, s2[k]);
                    }
                }
            }
        });
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
            const uint32_t to = channel_at<V>(a.channels, blockIdx.y * width + k);
            if (to >= a.channels) continue;
            float t = red[k];
            for (uint32_t q = 1; q < left; ++q) t += red[q * width + k];
            out[(uint64_t)which * a.channels + to] = t;
        }
    }
}

template <typename T, bool KEPT, int ACT, bool ONE>
__global__ __launch_bounds__(256) void k_groupnorm_backward_apply(co3_groupnorm_backward_args a, Slices cut, uint64_t first, const float *means)
{
    constexpr int V = kVec<T>;
    const uint64_t sample = first + blockIdx.z;
    const uint32_t rows = 256 / cut.packs, col = threadIdx.x % cut.packs, row = threadIdx.x / cut.packs;
    const Lane<V, ONE> lane(0, a.channels, (blockIdx.y * cut.packs + col) * V, row < rows);
    if (lane.n <= 0) return;
    const uint32_t end = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x + 1);
    Channels<V, ONE> ch;
    ch.load(a, sample, lane);
    float m1[ONE ? 1 : V] = {}, m2[ONE ? 1 : V] = {};
    for_groups(lane, 0, a.channels / a.groups, [&](int k, uint32_t g) {
        m1[k] = means[2 * (sample * a.groups + g)] * ch.rstd[k];
        m2[k] = means[2 * (sample * a.groups + g) + 1] * ch.rstd[k];
    });
    const Source<T, KEPT, ONE> source(a, sample, lane.base);
    const T *dy = static_cast<const T *>(a.dy) + sample * a.pixels * a.dy_stride + lane.base;
    T *dx = static_cast<T *>(a.dx) + sample * a.pixels * a.dx_stride + lane.base;
    with_rows<V, ONE>(a.channels, [&](auto full) {
        constexpr bool FULL = decltype(full)::value;
        for (uint32_t r = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x) + row; r < end; r += kAtOnce * rows) {
            typename Source<T, KEPT, ONE>::Raw raw[kAtOnce];
            typename Pack<T, V>::V d[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                raw[i] = source.template fetch<FULL>(r + i * rows, lane, r + i * rows < end);
                d[i] = load_lane<FULL>(dy + (r + i * rows) * a.dy_stride, lane, r + i * rows < end);
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                if (r + i * rows >= end) continue;
                const auto x = source.numbers(raw[i]);
                typename Pack<T, V>::V o;
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float xh = ch.xh(k, x[k]), dz = passed<ACT>((float)d[i][k], xh, ch.w[k], ch.b[k]);
                    o[k] = (T)ch.dx(k, xh, dz, m1[ONE ? 0 : k], m2[ONE ? 0 : k]);
                }
                store_lane<T, ONE>(dx + (r + i * rows) * a.dx_stride, lane, o);
            }
        }
    });
}

// m1 and m2 of a group, by the threads of a wavefront or of the workgroup.
template <int THREADS>
__device__ inline void mean_of_group(const co3_groupnorm_backward_args &a, uint32_t slices, uint64_t k, uint32_t thread, const float *partial, float *means)
{
    const uint64_t sample = k / a.groups;
    const uint32_t per = a.channels / a.groups, c0 = (uint32_t)(k % a.groups) * per;
    double s1 = 0.0, s2 = 0.0;
#pragma unroll 4
    for (uint32_t e = thread; e < slices * per; e += THREADS) {
        const uint32_t c = c0 + e % per;
        const float *p = partial + (sample * slices + e / per) * 2 * a.channels + c;
        const double w = a.weight ? a.weight[c] : 1.f;
        s1 += w * p[0];
        s2 += w * p[a.channels];
    }
    fold_two<THREADS>(s1, s2);
    if (thread) return;
    const double n = 1.0 / ((double)a.pixels * per);
    means[2 * k] = (float)(s1 * n);
    means[2 * k + 1] = (float)(s2 * n);
}

// What becomes of the sums of `parts` (samples, or slices of them) of each user, in fp64, since there may be thousands.  The first `grads`
// workgroups: 64 channels of either gradient of a user, a wavefront every sixteenth part.  The others: the means of a group each, or
// where there is little to add up (a wavefront took 44 us for 256 slices of 16 channels) of sixteen, a wavefront each.
static __global__ __launch_bounds__(1024) void k_groupnorm_grad(co3_groupnorm_backward_args a, uint64_t parts, uint64_t grads, uint32_t slices, uint64_t first,
                                                                const float *partial, float *means)
{
    __shared__ double part[16][64];
    const uint32_t lane = threadIdx.x & 63u, w = threadIdx.x >> 6, across = (2 * a.channels + 63) / 64;
    const uint64_t at = first + blockIdx.x;
    if (at >= grads) {
        const uint64_t all = a.U * a.samples_per_user * a.groups;
        if (few_terms(slices, a.channels / a.groups)) {
            const uint64_t k = (at - grads) * 16 + w;
            if (k < all) mean_of_group<64>(a, slices, k, lane, partial, means);
        } else if (at - grads < all) {
            mean_of_group<1024>(a, slices, at - grads, threadIdx.x, partial, means);
        }
        return;
    }
    const uint64_t u = at / across, c = at % across * 64 + lane, channels = a.channels;   // dbias's columns, then dweight's
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

template <typename T, bool KEPT>
static void backward_of(const co3_groupnorm_backward_args &a, hipStream_t s)
{
    const uint64_t samples = a.U * a.samples_per_user;
    const Whole w = whole_of(a.pixels, a.channels, a.groups, a.type, kBackward);
    float *partial = static_cast<float *>(a.workspace), *means = nullptr;
    const uint64_t grads = a.dweight || a.dbias ? (uint64_t)a.U * ((2 * a.channels + 63) / 64) : 0;
    uint64_t parts = a.samples_per_user, others = 0;
    Slices c = {};
    if (samples && w.threads) {
        ProfScope prof(K_GROUPNORM_BACKWARD, s);
        with_activation(a.activation, [&](auto act) {
            with_backward(w, [&](auto threads, auto held, auto one) {
                constexpr int WG = decltype(threads)::value, CH = decltype(held)::value;
                in_parts(samples, (uint64_t)WG * w.strip.blocks, ~0ull, [&](uint64_t first, uint32_t count) {
                    k_groupnorm_backward<T, KEPT, decltype(act)::value, WG, CH, decltype(one)::value>
                        <<<dim3(count, w.strip.blocks), dim3(WG), w.lds, s>>>(a, w.strip, first, grads ? partial : nullptr);
                });
            });
        });
    } else if (samples) {
        c = slices_of(samples, a.pixels, a.channels, a.type, kMostTerms);
        parts *= c.slices;
        others = few_terms(c.slices, a.channels / a.groups) ? (samples * a.groups + 15) / 16 : samples * a.groups;
        means = partial + up16(samples * c.slices * 2 * a.channels * sizeof(float)) / sizeof(float);
        ProfScope prof(K_GROUPNORM_SUMS, s);
        with_activation(a.activation, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            in_parts(samples, (uint64_t)256 * c.slices * c.columns, 65535, [&](uint64_t first, uint32_t count) {
                const dim3 grid(c.slices, c.columns, count);
                if (w.one) k_groupnorm_backward_sums<T, KEPT, ACT, true><<<grid, dim3(256), 0, s>>>(a, c, first, partial);
                else k_groupnorm_backward_sums<T, KEPT, ACT, false><<<grid, dim3(256), 0, s>>>(a, c, first, partial);
            });
        });
    }
    if (grads + others) {
        ProfScope prof(K_GROUPNORM_GRAD, s);
        in_parts(grads + others, 1024, ~0ull, [&](uint64_t first, uint32_t count) {
            k_groupnorm_grad<<<dim3(count), dim3(1024), 0, s>>>(a, parts, grads, c.slices, first, partial, means);
        });
    }
    if (!means) return;
    ProfScope prof(K_GROUPNORM_BACKWARD, s);
    with_activation(a.activation, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        in_parts(samples, (uint64_t)256 * c.slices * c.columns, 65535, [&](uint64_t first, uint32_t count) {
            const dim3 grid(c.slices, c.columns, count);
            if (w.one) k_groupnorm_backward_apply<T, KEPT, ACT, true><<<grid, dim3(256), 0, s>>>(a, c, first, means);
            else k_groupnorm_backward_apply<T, KEPT, ACT, false><<<grid, dim3(256), 0, s>>>(a, c, first, means);
        });
    });
}

template <bool KEPT>
static hipError_t launch_backward(const co3_groupnorm_backward_args &a, hipStream_t s)
{
    if (a.type == CO3_F32) backward_of<float, KEPT>(a, s);
    else if (a.type == CO3_BF16) backward_of<__bf16, KEPT>(a, s);
    else backward_of<_Float16, KEPT>(a, s);
    return hipGetLastError();
}

}  // namespace co3
