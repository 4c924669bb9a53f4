// What the kernels of group norm share (k_groupnorm.hip, groupnorm_backward.h).
#pragma once

#include <type_traits>

#include "blocks8.h"
#include "co3_internal.h"
#include "tensor_types.h"

namespace co3 {

struct Strip { uint32_t groups, blocks, packs; };   // groups of a workgroup, workgroups of a sample, packs of a pixel

// 1 / (1 + 2^(-z / ln 2)): exp2 and the reciprocal are good to a unit in the last place; 0 and 1 at the ends.  Two instructions at a quarter
// of the rate of others, where expf and a division are thirty: these kernels have some forty a value before they are bound by them.
__device__ inline float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504088896340736f)); }
template <int ACT>
__device__ inline float activated(float z) { return ACT == CO3_ACT_RELU ? (z > 0.f ? z : z != z ? z : 0.f) : ACT == CO3_ACT_SILU ? z * sigmoid(z) : z; }
// z.  ReLU's is rounded the same in both passes, by which they agree on its sign: a value has a gradient if and only if it is let through.
template <int ACT>
__device__ inline float argument(float x, float mean, float rstd, float w, float b)
{
    if (ACT != CO3_ACT_RELU) return __builtin_fmaf(x - mean, rstd * w, b);
    const float xh = (x - mean) * rstd;
    return xh * w + b;
}
// dy act'(z) of z = xh w + b.
template <int ACT>
__device__ inline float passed(float dy, float xh, float w, float b)
{
    if (ACT == CO3_ACT_NONE) return dy;
    if (ACT == CO3_ACT_RELU) return xh * w + b > 0.f ? dy : 0.f;   // of xh = (x - mean) rstd, as in argument()
    const float z = __builtin_fmaf(xh, w, b), p = sigmoid(z);
    return dy * __builtin_fmaf(p, __builtin_fmaf(-z, p, z), p);   // p (1 + z (1 - p))
}

// Waits for the loads of these numbers here.  Where branches of a thread's packs follow, the compiler waits in each of them again, for the stores of
// those in front too (128 x 256 x 60 fp32 with ReLU 8.1 us for 7.4, 256 x 1024 x 256 bf16 58.1 for 56.4).
template <int N, typename A>
__device__ inline void arrived(A &v)
{
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float f = v[k];
        asm volatile("" : "+v"(f));
        v[k] = f;
    }
}

// Sums of a pack's values and of their squares.
__device__ inline void add_pack(const Pack<float, 4>::V &p, float &s, float &q)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s += p[i];
        q = __builtin_fmaf(p[i], p[i], q);
    }
}
__device__ inline void add_pack(const Pack<__bf16, 8>::V &p, float &s, float &q)   // two products and a sum an instruction
{
    typedef __bf16 two __attribute__((ext_vector_type(2)));
    const two one = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const two v = {p[2 * i], p[2 * i + 1]};
        s = __builtin_amdgcn_fdot2_f32_bf16(v, one, s, false);
        q = __builtin_amdgcn_fdot2_f32_bf16(v, v, q, false);
    }
}
__device__ inline void add_pack(const Pack<_Float16, 8>::V &p, float &s, float &q)
{
    typedef _Float16 two __attribute__((ext_vector_type(2)));
    const two one = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const two v = {p[2 * i], p[2 * i + 1]};
        s = __builtin_amdgcn_fdot2(v, one, s, false);
        q = __builtin_amdgcn_fdot2(v, v, q, false);
    }
}

// A thread's pack of a strip of channels c0 .. c0 + cn: V channels from `base` on, of which those from `low` up to `n` are its own; n = 0: none.  The
// strip's last pack lies back within the pixel where it would reach beyond the strip, over channels of the pack in front, so that it is one load.
template <int V, bool WHOLE>
struct Lane {
    uint32_t base;
    int low, n;
    __device__ inline Lane(uint32_t c0, uint32_t cn, uint32_t j, bool there)
    {
        const uint32_t end = c0 + cn;
        base = c0 + j;
        low = 0;
        n = there && j < cn ? V : 0;
        if (WHOLE || n == 0 || j + V <= cn) return;
        if (end >= (uint32_t)V) {
            low = (int)(j + V - cn);
            base = end - V;
        } else {
            n = (int)(cn - j);   // a row of fewer than V channels
        }
    }
    __device__ inline bool own(int k) const { return WHOLE ? n > 0 : k >= low && k < n; }
};
// Where channel c of a strip is among its packs' V channels each.
template <int V>
__device__ inline uint32_t place_of(uint32_t c0, uint32_t cn, uint32_t c) { return c < cn / V * V || c0 + cn < (uint32_t)V ? c : c + V - cn % V; }

// FULL: the pixels have as many channels as a pack, or more: a pack is one load, or none.
template <bool FULL, typename T, bool WHOLE>
__device__ inline typename Pack<T, kVec<T>>::V load_lane(const T *row, const Lane<kVec<T>, WHOLE> &lane, bool there)
{
    constexpr int V = kVec<T>, H = V / 2;
    if constexpr (FULL) {
        return load_pack<T, V>(row, there && lane.n > 0 ? V : 0);
    } else {
        typename Pack<T, V>::V v;
        const int n = there ? lane.n : 0;
        const auto low = load_pack<T, H>(row, n), high = load_pack<T, H>(row + H, n - H);
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = k < H ? low[k < H ? k : 0] : high[k < H ? 0 : k - H];
        return v;
    }
}
// f(whether they are FULL), by a branch of all threads.
template <int V, bool WHOLE, typename F>
__device__ inline void with_rows(uint32_t channels, F &&f)
{
    if (WHOLE || channels >= (uint32_t)V) f(std::true_type());
    else f(std::integral_constant<bool, WHOLE>());
}
template <typename T, bool WHOLE>
__device__ inline void store_lane(T *row, const Lane<kVec<T>, WHOLE> &lane, const typename Pack<T, kVec<T>>::V &v)
{
    constexpr int V = kVec<T>;
    if (WHOLE || (lane.low == 0 && lane.n == V)) {
        store_pack<T, V>(row, V, v);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (lane.own(k)) row[k] = v[k];
    }
}

// f(k, the group of channel k within a strip from c0 on) for the channels that are a thread's own; WHOLE: for the first, whose group is that of all.
template <int V, bool WHOLE, typename F>
__device__ inline void for_groups(const Lane<V, WHOLE> &lane, uint32_t c0, uint32_t per, F &&f)
{
    const uint32_t c = lane.base + (uint32_t)lane.low - c0;
    uint32_t g = lane.n > 0 ? c / per : 0, r = c - g * per;
#pragma unroll
    for (int k = 0; k < (WHOLE ? 1 : V); ++k) {
        if (!lane.own(k)) continue;
        f(k, g);
        if (++r == per) {
            r = 0;
            ++g;
        }
    }
}

// Sums of a workgroup's threads whose numbers are equal modulo `packs`, a power of two: red[c], c = pack V + channel, has those of
// `s`, red[packs V + c] those of `q`.  Up to 16 packs a wavefront's lanes are added up first: half of the values go to the other half
// of the lanes at each of two steps, so that these take as many additions as there are values.
template <int V, int WG>
__device__ inline void fold_channels(const float (&s)[V], const float (&q)[V], float *red, uint32_t packs)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x / 64, width = packs * V;
    float *parts = red + 2 * width;
    uint32_t count = WG / 64;
    if (packs <= 16) {
        float t[V], u[V / 2];
#pragma unroll
        for (int k = 0; k < V; ++k) {   // lanes 0 to 31 go on with s, the others with q
            const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(s[k]), __float_as_uint(q[k]), false, false);
            t[k] = __uint_as_float(p[0]) + __uint_as_float(p[1]);
        }
#pragma unroll
        for (int k = 0; k < V / 2; ++k) {   // every other sixteen lanes with the second half of the channels
            const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(t[k]), __float_as_uint(t[k + V / 2]), false, false);
            u[k] = __uint_as_float(p[0]) + __uint_as_float(p[1]);
            for (uint32_t o = 8; o >= packs; o >>= 1) u[k] += __shfl_xor(u[k], o);
        }
        if (lane % 16 < packs) {
#pragma unroll
            for (int k = 0; k < V / 2; ++k) parts[wave * 2 * width + lane / 32 * width + lane % 16 * V + lane / 16 % 2 * (V / 2) + k] = u[k];
        }
    } else {
        const uint32_t row = threadIdx.x / packs, col = threadIdx.x % packs;
        count = WG / packs;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            parts[row * 2 * width + col * V + k] = s[k];
            parts[row * 2 * width + width + col * V + k] = q[k];
        }
    }
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < 2 * width; c += WG) {
        float f = parts[c];
        for (uint32_t w = 1; w < count; ++w) f += parts[w * 2 * width + c];
        red[c] = f;
    }
    __syncthreads();
}

// f(g, sum, sum) by one thread for every group, of what `term(place, channel)` gives of its channels: eight threads add up a group's, or a
// wavefront where there are many.
template <int WG, int V, typename S, typename Term, typename F>
__device__ inline void fold_groups(uint32_t groups, uint32_t per, uint32_t c0, uint32_t cn, Term &&term, F &&f)
{
    const uint32_t together = per > 64 ? 64 : 8;
    for (uint32_t k = threadIdx.x; k < groups * together; k += WG) {   // those of a group go round together
        const uint32_t g = k / together;
        S s = 0, q = 0;
        for (uint32_t c = g * per + k % together; c < (g + 1) * per; c += together) term(place_of<V>(c0, cn, c), c, s, q);
        for (uint32_t o = together / 2; o; o >>= 1) {
            s += __shfl_xor(s, o);
            q += __shfl_xor(q, o);
        }
        if (k % together == 0) f(g, s, q);
    }
    __syncthreads();
}

// Workgroups of 256 threads: `packs` of them next to each other in a pixel, so many columns of these, slices of the pixels.
struct Slices { uint32_t packs, columns, slices; };

__device__ inline uint32_t slice_begin(uint32_t pixels, uint32_t slices, uint32_t i) { return (uint32_t)((uint64_t)pixels * i / slices); }

// The channel at a place among a pixel's packs; one that is not there for places that another pack has.
template <int V>
__device__ inline uint32_t channel_at(uint32_t channels, uint32_t place)
{
    if (place < channels / V * V || channels < (uint32_t)V) return place;
    const uint32_t back = V - channels % V;
    return place % V < back ? ~0u : place - back;
}

// Two sums of all threads of a workgroup.
template <int WG>
__device__ inline void fold_two(double &s, double &q)
{
    __shared__ double red[WG / 64][2];
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        s += __shfl_xor(s, o);
        q += __shfl_xor(q, o);
    }
    if (WG == 64) return;
    if (threadIdx.x % 64 == 0) {
        red[threadIdx.x / 64][0] = s;
        red[threadIdx.x / 64][1] = q;
    }
    __syncthreads();
    s = red[0][0];
    q = red[0][1];
#pragma unroll
    for (int k = 1; k < WG / 64; ++k) {
        s += red[k][0];
        q += red[k][1];
    }
}

// Whether a wavefront adds up a group's sums of so many slices, or a workgroup of sixteen.
__host__ __device__ inline bool few_terms(uint32_t slices, uint32_t per) { return (uint64_t)slices * per <= 512; }

// ---- launches -----------------------------------------------------------------------------------------------

static inline uint32_t elements_of_pack(int32_t type) { return type == CO3_F32 ? 4 : 8; }

// One launch: groups of `wide` packs of a pixel or more to a workgroup, the first of the forms that holds them.  threads = 0: none does.
struct Form { uint32_t threads, held, wide; };                         // `held` packs a thread
struct Whole { Strip strip; uint32_t threads, held, lds; bool one; };  // one: packs lie within groups
template <size_t N>
static Whole whole_of(uint64_t pixels, uint32_t channels, uint32_t groups, int32_t type, const Form (&forms)[N])
{
    const uint32_t V = elements_of_pack(type), per = channels / groups;
    Whole w = {};
    w.one = per % V == 0;
    for (const Form &f : forms) {
        w.strip.groups = (f.wide * V + per - 1) / per;
        if (w.strip.groups > groups) w.strip.groups = groups;
        w.strip.blocks = (groups + w.strip.groups - 1) / w.strip.groups;
        w.strip.packs = 1;
        while (w.strip.packs * V < w.strip.groups * per) w.strip.packs *= 2;
        if (!w.one && f.threads * f.held > 4096) continue;   // they would spill
        if (f.threads / w.strip.packs * (uint64_t)f.held < pixels) continue;
        const uint32_t parts = w.strip.packs <= 16 ? f.threads / 64 : f.threads / w.strip.packs;
        const uint32_t channel_sums = (1 + parts) * 2 * w.strip.packs * V, sums = channel_sums > 2 * f.threads ? channel_sums : 2 * f.threads;
        w.lds = (sums + 2 * w.strip.groups) * (uint32_t)sizeof(float);   // of the channels, or of the threads; two numbers of every group
        if (w.lds > 65536) continue;
        w.threads = f.threads;
        w.held = f.held;
        break;
    }
    return w;
}

static Slices slices_of(uint64_t samples, uint64_t pixels, uint32_t channels, int32_t type, uint64_t most_terms)
{
    Slices s;
    const uint32_t packs = (channels + elements_of_pack(type) - 1) / elements_of_pack(type);
    s.columns = (packs + 31) / 32;
    s.packs = (packs + s.columns - 1) / s.columns;
    const uint32_t rows = 256 / s.packs;
    const uint64_t fill = (2048 + samples * s.columns - 1) / (samples * s.columns), room = (pixels + 8 * rows - 1) / (8 * rows);
    uint64_t n = fill < room ? fill : room;
    const uint64_t least = (pixels + rows * most_terms - 1) / (rows * most_terms);
    if (n < least) n = least;
    s.slices = (uint32_t)(n < 1 ? 1 : n);
    return s;
}

static inline size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }
constexpr Form kForward[] = {{64, 1, 8}, {64, 4, 8}, {256, 4, 8}, {512, 8, 8}, {512, 16, 8}}, kBackward[] = {{64, 1, 8}, {64, 4, 8}, {256, 4, 8}, {512, 8, 8}, {512, 8, 4}, {1024, 8, 8}};
constexpr int kAtOnce = 4;   // packs of a thread on their way at a time, by slices
constexpr uint64_t kNoLimit = 1ull << 31, kMostTerms = 512;

// A launch of HIP has fewer than 2^32 threads: `threads` for each of `count`, at most `at_once` of them in one.
template <typename F>
static void in_parts(uint64_t count, uint64_t threads, uint64_t at_once, F &&launch)
{
    const uint64_t room = ((1ull << 32) - 1) / threads, most = room == 0 ? 1 : room < at_once ? room : at_once;   // 0: a launch that is refused
    for (uint64_t i = 0; i < count; i += most) launch(i, (uint32_t)(count - i < most ? count - i : most));
}

template <typename F>
static void with_activation(int32_t activation, F &&f)
{
    if (activation == CO3_ACT_RELU) f(std::integral_constant<int, CO3_ACT_RELU>());
    else if (activation == CO3_ACT_SILU) f(std::integral_constant<int, CO3_ACT_SILU>());
    else f(std::integral_constant<int, CO3_ACT_NONE>());
}

// f(threads, packs held, one) of a form.
template <uint32_t THREADS, uint32_t HELD, typename F>
static bool if_form(const Whole &w, F &&f)
{
    if (w.threads != THREADS || w.held != HELD) return false;
    const std::integral_constant<int, THREADS> threads;
    const std::integral_constant<int, HELD> held;
    if (w.one) f(threads, held, std::true_type());
    else if constexpr (THREADS * HELD <= 4096) f(threads, held, std::false_type());
    return true;
}
template <typename F>
static void with_forward(const Whole &w, F &&f)
{
    if_form<64, 1>(w, f) || if_form<64, 4>(w, f) || if_form<256, 4>(w, f) || if_form<512, 8>(w, f) || if_form<512, 16>(w, f);
}
template <typename F>
static void with_backward(const Whole &w, F &&f)
{
    if_form<64, 1>(w, f) || if_form<64, 4>(w, f) || if_form<256, 4>(w, f) || if_form<512, 8>(w, f) || if_form<1024, 8>(w, f);
}

}  // namespace co3
