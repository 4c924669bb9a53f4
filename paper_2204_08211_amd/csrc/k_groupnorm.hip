// Group norm with an activation, channels last: forward pass, backward pass, the weight's gradients per user.
//
// Forward:   mean, var over a sample's pixels and a group's channels, rstd = 1 / sqrt(var + eps), z = (x - mean) rstd w + b, y = act(z)
// Backward:  xh = (x - mean) rstd,  z = xh w + b,  dz = dy act'(z).  Of every sample and channel
//            S1 = sum over the pixels of dz,  S2 = sum of dz xh;  over a group's channels m1 = mean(w S1), m2 = mean(w S2):
//            dx = rstd (dz w - m1 - xh m2),  dweight[u] = sum over the user's samples of S2,  dbias[u] = of S1
// so one pass over the data gives all sums, and a second one dx.
//
// Two ways.  Where a workgroup can hold a sample's pixels of some whole groups (64 or 128 bytes of a pixel, or more) in registers, it reads them once
// and all is one launch.  Beyond that the sums of slices of pixels go through the workspace, and x (and dy) are read twice.
// All sums are formed in a fixed order.
//
// Measured (MI355X, a large copy runs at 4.8 TB/s; kernels): forward 256 x 1024 x 256 bf16 with SiLU 63 to 68 us = 4.3 to 3.9 TB/s; 8 x 16384 x 256 by slices
// 22 + 6 + 24 us.  Backward of 128 x 1024 x 256 bf16 from x in 8 bits 59 us with SiLU, where vector instructions fill 72 % of the cycles (dz is made twice,
// since the registers hold x and dy), 48 without an activation; 5 more for the users' gradients.  4 x 16384 x 512 by slices 38 + 6 + 34 us.
// Groups of 15 channels, 128 x 1024 x 60 fp32, by slices 14 + 4.5 + 17 us (41 + 5 in one launch, of partial packs).
#include "groupnorm.h"

namespace co3 {

// ---- in one launch ------------------------------------------------------------------------------------------

// mean and rstd of a workgroup's groups into its LDS.
// The sums of x and of its squares do while no group's mean is more than twice its spread: formed in fp32 over a thread's packs (of partial ones
// over the workgroup's threads too), with at most 128 terms one behind the other, and in fp64 beyond, each is off by at most 128 2^-24 of its
// terms' sizes, and the variance, their difference, by five times that.  Otherwise the distances from the mean, and their squares, are
// added up in a second turn, and where squares leave fp32 at either end, those of x times a power of two, which rounds nothing.  That mean
// is an fp32 number near the group's, off by e; the distances' mean says how far, and its square leaves the variance: off by at most 32 2^-24 (1 + 2 (e / spread)^2)
// of itself, whatever the mean.
template <typename T, int WG, int CH, bool ONE>
__device__ inline void statistics(const co3_groupnorm_args &a, const typename Pack<T, kVec<T>>::V (&p)[CH], float *red, float *mean, float *rstd,
                                  uint32_t rows, uint32_t packs, uint32_t row, uint32_t c0, uint32_t cn, uint32_t groups, uint32_t per, const Lane<kVec<T>, ONE> &lane)
{
    constexpr int V = kVec<T>;
    const uint32_t pixels = (uint32_t)a.pixels, width = packs * V;
    const double scale = 1.0 / ((double)pixels * (double)per);
    const auto decide = [&](uint32_t g, double s, double q) {
        const double m = s * scale, var = q * scale - m * m;
        const bool large = !(q < 1e37), small = q * scale < 1e-24 && a.eps < 1e-17f;   // large: also what is not finite
        mean[g] = (float)m;
        rstd[g] = large ? -0x1p-80f : small ? -0x1p80f : m * m <= 4.0 * var ? (float)(1.0 / sqrt(var + (double)a.eps)) : -1.f;   // below 0: the power of two
    };
    if constexpr (ONE) {   // a thread has one group's
        float s = 0.f, q = 0.f;
#pragma unroll
        for (int i = 0; i < CH; ++i) add_pack(p[i], s, q);   // zeros beyond the pixels
        red[2 * threadIdx.x] = s;
        red[2 * threadIdx.x + 1] = q;
        __syncthreads();
        const uint32_t each = per / V;   // packs of a group in a pixel
        for (uint32_t g = threadIdx.x / 64; g < groups; g += WG / 64) {
            double ds = 0.0, dq = 0.0;
            for (uint32_t k = threadIdx.x % 64; k < rows * each; k += 64) {
                const uint32_t at = 2 * (k / each * packs + g * each + k % each);
                ds += red[at];
                dq += red[at + 1];
            }
#pragma unroll
            for (int o = 32; o; o >>= 1) {
                ds += __shfl_xor(ds, o);
                dq += __shfl_xor(dq, o);
            }
            if (threadIdx.x % 64 == 0) decide(g, ds, dq);
        }
        __syncthreads();
    } else {
        float s[V], q[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            s[k] = q[k] = 0.f;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const float v = (float)p[i][k];
                s[k] += v;
                q[k] = __builtin_fmaf(v, v, q[k]);
            }
            if (!lane.own(k)) s[k] = q[k] = 0.f;
        }
        fold_channels<V, WG>(s, q, red, packs);
        fold_groups<WG, V, double>(groups, per, c0, cn, [&](uint32_t at, uint32_t, double &ds, double &dq) {
            ds += red[at];
            dq += red[width + at];
        }, decide);
    }
    bool again = false, large = false;
    for (uint32_t g = 0; g < groups; ++g) {
        again = again || rstd[g] < 0.f;
        large = large || rstd[g] == -0x1p-80f;
    }
    if (!again) return;
    const auto power = [&](uint32_t g) { return rstd[g] < 0.f ? -rstd[g] : 1.f; };
    float s[V], none[V], m[ONE ? 1 : V] = {}, f[ONE ? 1 : V] = {};
    for_groups(lane, c0, per, [&](int k, uint32_t g) { f[k] = power(g); });
    __syncthreads();   // all have seen the groups'
    if (large) {       // their sums may have left fp32 too
#pragma unroll
        for (int k = 0; k < V; ++k) {
            s[k] = none[k] = 0.f;
            if (!lane.own(k)) continue;
#pragma unroll
            for (int i = 0; i < CH; ++i) s[k] += (float)p[i][k] * f[ONE ? 0 : k];   // zeros beyond the pixels
        }
        fold_channels<V, WG>(s, none, red, packs);
        fold_groups<WG, V, double>(groups, per, c0, cn, [&](uint32_t at, uint32_t, double &ds, double &) { ds += red[at]; },
                                   [&](uint32_t g, double ds, double) { mean[g] = rstd[g] == -0x1p-80f ? (float)(ds * scale * 0x1p80) : mean[g]; });
    }
    for_groups(lane, c0, per, [&](int k, uint32_t g) { m[k] = mean[g]; });
    float off[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        s[k] = off[k] = 0.f;
        if (!lane.own(k)) continue;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const float v = __builtin_fmaf((float)p[i][k], f[ONE ? 0 : k], -m[ONE ? 0 : k] * f[ONE ? 0 : k]), d = row + i * rows < pixels ? v : 0.f;
            s[k] = __builtin_fmaf(d, d, s[k]);
            off[k] += d;
        }
    }
    fold_channels<V, WG>(s, off, red, packs);
    fold_groups<WG, V, double>(groups, per, c0, cn, [&](uint32_t at, uint32_t, double &ds, double &dd) {
        ds += red[at];
        dd += red[width + at];
    }, [&](uint32_t g, double ds, double dd) {
        const double t = power(g), e = dd * scale, var = ds * scale - e * e;
        if (fabs(e) < INFINITY) mean[g] = (float)((double)mean[g] + e / t);   // an infinite mean stays
        rstd[g] = (float)(1.0 / sqrt((var > 0.0 ? var : var != var ? var : 0.0) / (t * t) + (double)a.eps));
    });
}

template <typename T, int ACT, int WG, int CH, bool ONE>
__global__ __launch_bounds__(WG, 4) void k_groupnorm(co3_groupnorm_args a, Strip strip, uint64_t first)
{
    constexpr int V = kVec<T>;
    extern __shared__ float red[];   // the groups' mean and rstd, then what the sums take
    const uint64_t sample = first + blockIdx.x;
    const uint32_t per = a.channels / a.groups, g0 = blockIdx.y * strip.groups, c0 = g0 * per;
    const uint32_t groups = a.groups - g0 < strip.groups ? a.groups - g0 : strip.groups, cn = groups * per;
    const uint32_t rows = WG / strip.packs, row = threadIdx.x / strip.packs, pixels = (uint32_t)a.pixels;
    float *mean = red, *rstd = mean + strip.groups;
    const Lane<V, ONE> lane(c0, cn, threadIdx.x % strip.packs * V, true);
    const T *x = static_cast<const T *>(a.x) + sample * a.pixels * a.x_stride + lane.base;
    typename Pack<T, V>::V p[CH];
    with_rows<V, ONE>(a.channels, [&](auto full) {
#pragma unroll
        for (int i = 0; i < CH; ++i) p[i] = load_lane<decltype(full)::value>(x + (row + i * rows) * a.x_stride, lane, row + i * rows < pixels);
    });
    statistics<T, WG, CH, ONE>(a, p, red + 2 * strip.groups, mean, rstd, rows, strip.packs, row, c0, cn, groups, per, lane);
    if (threadIdx.x < groups) {
        const uint64_t at = sample * a.groups + g0 + threadIdx.x;
        if (a.mean) a.mean[at] = mean[threadIdx.x];
        if (a.rstd) a.rstd[at] = rstd[threadIdx.x];
    }
    if (lane.n <= 0) return;
    float m[ONE ? 1 : V] = {}, f[ONE ? 1 : V] = {};
    typename Pack<float, V>::V w, b;
#pragma unroll
    for (int k = 0; k < V; ++k) { w[k] = 1.f; b[k] = 0.f; }
    if (a.weight) w = load_pack<float, V>(a.weight + lane.base, ONE ? V : lane.n);
    if (a.bias) b = load_pack<float, V>(a.bias + lane.base, ONE ? V : lane.n);
    for_groups(lane, c0, per, [&](int k, uint32_t g) {
        m[k] = mean[g];
        f[k] = rstd[g];
    });
    arrived<V>(w);
    arrived<V>(b);
    T *y = static_cast<T *>(a.y) + sample * a.pixels * a.y_stride + lane.base;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const uint32_t r = row + i * rows;
        if (r >= pixels) continue;
        typename Pack<T, V>::V o;
#pragma unroll
        for (int k = 0; k < V; ++k) o[k] = (T)activated<ACT>(argument<ACT>((float)p[i][k], m[ONE ? 0 : k], f[ONE ? 0 : k], w[k], b[k]));
        store_lane<T, ONE>(y + r * a.y_stride, lane, o);
    }
}

// ---- by slices of pixels ------------------------------------------------------------------------------------

// What a group's distances are taken from: its first value, or 0 where that is not finite.
__device__ inline float taken_from(float first) { return fabsf(first) < INFINITY ? first : 0.f; }

// Those of a thread's channels (WHOLE: of the first).  All loads before the first one is looked at, without a branch between them.
template <typename T, bool WHOLE>
__device__ inline void first_values(const T *sample, uint32_t per, const Lane<kVec<T>, WHOLE> &lane, float *from)
{
    constexpr int N = WHOLE ? 1 : kVec<T>;
    const uint32_t c = lane.n > 0 ? lane.base : 0;
    uint32_t g = c / per, r = c - g * per;
    T v[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        v[k] = sample[k < lane.n ? g * per : 0];
        r = r + 1 == per ? 0 : r + 1;
        g += r == 0 ? 1 : 0;
    }
#pragma unroll
    for (int k = 0; k < N; ++k) from[k] = taken_from((float)v[k]);
}

// Sums of the distances from a value of the group, and of their squares, in fp64, where no finite input overflows.  Any of n values is at most
// sqrt(n) times the spread away from the mean, so whatever the mean is, the variance, a difference, is off by some n 2^-53 of itself at most.
template <typename T, bool ONE>
__global__ __launch_bounds__(256) void k_groupnorm_sums(co3_groupnorm_args a, Slices cut, uint64_t first, double *partial)
{
    constexpr int V = kVec<T>;
    __shared__ double red[256 * V];
    const uint64_t sample = first + blockIdx.z;
    const uint32_t rows = 256 / cut.packs, col = threadIdx.x % cut.packs, row = threadIdx.x / cut.packs, width = cut.packs * V;
    const Lane<V, ONE> lane(0, a.channels, (blockIdx.y * cut.packs + col) * V, row < rows);
    const uint32_t end = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x + 1), per = a.channels / a.groups;
    const T *all = static_cast<const T *>(a.x) + sample * a.pixels * a.x_stride, *x = all + lane.base;
    double s[V], q[V];
    float from[ONE ? 1 : V];
    first_values(all, per, lane, from);
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = q[k] = 0.0;
    if (lane.n > 0) {
        with_rows<V, ONE>(a.channels, [&](auto full) {
            for (uint32_t r = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x) + row; r < end; r += kAtOnce * rows) {
                typename Pack<T, V>::V p[kAtOnce];
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) p[i] = load_lane<decltype(full)::value>(x + (r + i * rows) * a.x_stride, lane, r + i * rows < end);
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    if (r + i * rows >= end) continue;
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        const double v = (double)(float)p[i][k] - (double)from[ONE ? 0 : k];
                        s[k] += v;
                        q[k] = __builtin_fma(v, v, q[k]);
                    }
                }
            }
        });
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
            const uint32_t to = channel_at<V>(a.channels, blockIdx.y * width + k);
            if (to >= a.channels) continue;
            double t = red[k];
            for (uint32_t r = 1; r < rows; ++r) t += red[r * width + k];
            out[(uint64_t)which * a.channels + to] = t;
        }
    }
}

// mean and rstd of a group, a workgroup each: of one wavefront where there is little to add up, otherwise of sixteen.
template <typename T, int WG>
__global__ __launch_bounds__(WG) void k_groupnorm_stats(co3_groupnorm_args a, uint32_t slices, uint64_t first, const double *partial, float *mean, float *rstd)
{
    const uint64_t k = first + blockIdx.x, sample = k / a.groups;
    const uint32_t per = a.channels / a.groups, c0 = (uint32_t)(k % a.groups) * per;
    double s = 0.0, q = 0.0;
#pragma unroll 4
    for (uint32_t e = threadIdx.x; e < slices * per; e += WG) {
        const double *p = partial + (sample * slices + e / per) * 2 * a.channels + c0 + e % per;
        s += p[0];
        q += p[a.channels];
    }
    fold_two<WG>(s, q);
    if (threadIdx.x) return;
    const double n = 1.0 / ((double)a.pixels * per), m = s * n, var = q * n - m * m;
    mean[k] = (float)((double)taken_from((float)static_cast<const T *>(a.x)[sample * a.pixels * a.x_stride + c0]) + m);
    rstd[k] = (float)(1.0 / sqrt((var > 0.0 ? var : var != var ? var : 0.0) + (double)a.eps));
}

template <typename T, int ACT>
__global__ __launch_bounds__(256) void k_groupnorm_apply(co3_groupnorm_args a, Slices cut, uint64_t first, const float *mean, const float *rstd)
{
    constexpr int V = kVec<T>;
    const uint64_t sample = first + blockIdx.z;
    const uint32_t rows = 256 / cut.packs, col = threadIdx.x % cut.packs, row = threadIdx.x / cut.packs;
    const Lane<V, false> lane(0, a.channels, (blockIdx.y * cut.packs + col) * V, row < rows);
    if (lane.n <= 0) return;
    const uint32_t end = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x + 1), per = a.channels / a.groups;
    float m[V], f[V];
    typename Pack<float, V>::V w, b;
#pragma unroll
    for (int k = 0; k < V; ++k) { m[k] = f[k] = 0.f; w[k] = 1.f; b[k] = 0.f; }
    if (a.weight) w = load_pack<float, V>(a.weight + lane.base, lane.n);
    if (a.bias) b = load_pack<float, V>(a.bias + lane.base, lane.n);
    for_groups(lane, 0, per, [&](int k, uint32_t g) {
        m[k] = mean[sample * a.groups + g];
        f[k] = rstd[sample * a.groups + g];
    });
    const T *x = static_cast<const T *>(a.x) + sample * a.pixels * a.x_stride + lane.base;
    T *y = static_cast<T *>(a.y) + sample * a.pixels * a.y_stride + lane.base;
    with_rows<V, false>(a.channels, [&](auto full) {
        for (uint32_t r = slice_begin((uint32_t)a.pixels, cut.slices, blockIdx.x) + row; r < end; r += kAtOnce * rows) {
            typename Pack<T, V>::V p[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) p[i] = load_lane<decltype(full)::value>(x + (r + i * rows) * a.x_stride, lane, r + i * rows < end);
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                if (r + i * rows >= end) continue;
                typename Pack<T, V>::V o;
#pragma unroll
                for (int k = 0; k < V; ++k) o[k] = (T)activated<ACT>(argument<ACT>((float)p[i][k], m[k], f[k], w[k], b[k]));
                store_lane<T, false>(y + (r + i * rows) * a.y_stride, lane, o);
            }
        }
    });
}

// ---- launches -----------------------------------------------------------------------------------------------

size_t groupnorm_workspace_bytes(uint64_t samples, uint64_t pixels, uint32_t channels, uint32_t groups, int32_t type)
{
    if (samples == 0 || whole_of(pixels, channels, groups, type, kForward).threads) return 0;
    const Slices c = slices_of(samples, pixels, channels, type, kNoLimit);
    return samples * c.slices * 2 * channels * sizeof(double) + 2 * up16(samples * groups * sizeof(float));
}

size_t groupnorm_backward_workspace_bytes(uint32_t U, uint64_t samples_per_user, uint64_t pixels, uint32_t channels, uint32_t groups, int32_t type)
{
    const uint64_t samples = U * samples_per_user;
    if (samples == 0) return 0;
    if (whole_of(pixels, channels, groups, type, kBackward).threads) return samples * 2 * channels * sizeof(float);
    const Slices c = slices_of(samples, pixels, channels, type, kMostTerms);
    return up16(samples * c.slices * 2 * channels * sizeof(float)) + samples * groups * 2 * sizeof(float);
}

template <typename T>
static void forward_of(const co3_groupnorm_args &a, hipStream_t s)
{
    const Whole w = whole_of(a.pixels, a.channels, a.groups, a.type, kForward);
    if (w.threads) {
        ProfScope prof(K_GROUPNORM, s);
        with_activation(a.activation, [&](auto act) {
            with_forward(w, [&](auto threads, auto held, auto one) {
                constexpr int WG = decltype(threads)::value, CH = decltype(held)::value;
                in_parts(a.samples, (uint64_t)WG * w.strip.blocks, ~0ull, [&](uint64_t first, uint32_t count) {
                    k_groupnorm<T, decltype(act)::value, WG, CH, decltype(one)::value>
                        <<<dim3(count, w.strip.blocks), dim3(WG), w.lds, s>>>(a, w.strip, first);
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
            const dim3 grid(c.slices, c.columns, count);
            if (w.one) k_groupnorm_sums<T, true><<<grid, dim3(256), 0, s>>>(a, c, first, partial);
            else k_groupnorm_sums<T, false><<<grid, dim3(256), 0, s>>>(a, c, first, partial);
        });
        const bool few = few_terms(c.slices, a.channels / a.groups);
        in_parts(a.samples * a.groups, few ? 64 : 1024, ~0ull, [&](uint64_t first, uint32_t count) {
            if (few) k_groupnorm_stats<T, 64><<<dim3(count), dim3(64), 0, s>>>(a, c.slices, first, partial, mean, rstd);
            else k_groupnorm_stats<T, 1024><<<dim3(count), dim3(1024), 0, s>>>(a, c.slices, first, partial, mean, rstd);
        });
    }
    ProfScope prof(K_GROUPNORM, s);
    with_activation(a.activation, [&](auto act) {
        in_parts(a.samples, (uint64_t)256 * c.slices * c.columns, 65535, [&](uint64_t first, uint32_t count) {
            k_groupnorm_apply<T, decltype(act)::value><<<dim3(c.slices, c.columns, count), dim3(256), 0, s>>>(a, c, first, mean, rstd);
        });
    });
}

hipError_t launch_groupnorm(const co3_groupnorm_args &a, hipStream_t s)
{
    if (a.type == CO3_F32) forward_of<float>(a, s);
    else if (a.type == CO3_BF16) forward_of<__bf16>(a, s);
    else forward_of<_Float16>(a, s);
    return hipGetLastError();
}

}  // namespace co3
