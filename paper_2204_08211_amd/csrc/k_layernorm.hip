// Layer norm: forward pass, backward pass, the reduction of the weight's gradients per user.
//
// Forward:   mean, var of a row, rstd = 1 / sqrt(var + eps), y = (x - mean) rstd weight + bias
// Backward:  t = dy weight, xh = (x - mean) rstd, dx = rstd (t - mean(t) - xh mean(t xh)),
//            dweight[u] = sum over the rows of user u of dy xh, dbias[u] = sum of dy
// Both are bound by memory: every element is read once and written once, the row stays in registers in between.  All
// sums are fp32 over a lane's elements and then over the lanes in a fixed order; the variance is the mean of the squared
// distances from the mean, which a mean far larger than the spread does not harm.
//
// Measured (MI355X, a large copy runs at 4.8 TB/s): forward 16384 x 4096 bf16 58 us = 4.6 TB/s; backward 16384 x 8192 bf16 175 us =
// 4.6 TB/s, eight users' 1024 x 1001 fp32 29 us = 3.4 TB/s (24 us, and 4 us for the sums of the slices).
#include "co3_internal.h"
#include "tensor_types.h"

namespace co3 {

// TPR threads share a row: TPR <= 64 lanes of a wavefront, or the whole workgroup.  A thread holds CH packs of 16 bytes,
// the packs of neighbouring threads next to each other.
template <int TPR>
__device__ inline float row_sum(float v, float *lds)
{
#pragma unroll
    for (int o = (TPR < 64 ? TPR : 64) / 2; o; o >>= 1) v += __shfl_xor(v, o);
    if (TPR > 64) {
        const int w = threadIdx.x >> 6;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[w] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int i = 1; i < TPR / 64; ++i) v += lds[i];
    }
    return v;
}

// Two sums with one meeting of the workgroup: rows take the two places in turn, so that nobody waits for the readers of the row before.
template <int TPR>
__device__ inline void row_sums(float &v, float &u, float (*lds)[2])
{
#pragma unroll
    for (int o = (TPR < 64 ? TPR : 64) / 2; o; o >>= 1) {
        v += __shfl_xor(v, o);
        u += __shfl_xor(u, o);
    }
    if (TPR > 64) {
        const int w = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            lds[w][0] = v;
            lds[w][1] = u;
        }
        __syncthreads();
        v = lds[0][0];
        u = lds[0][1];
#pragma unroll
        for (int i = 1; i < TPR / 64; ++i) {
            v += lds[i][0];
            u += lds[i][1];
        }
    }
}

// A row stays in registers between its sums and its result.  Few lanes a row where rows are short, so that a load brings many of them; one
// wavefront up to 512 packs, which needs no meeting; a workgroup beyond.
template <typename T, int TPR, int CH>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_layernorm(co3_layernorm_args a)
{
    constexpr int V = kVec<T>, WG = TPR > 256 ? TPR : 256;
    __shared__ float lds[WG / 64];
    const uint64_t row = (uint64_t)blockIdx.x * (WG / TPR) + threadIdx.x / TPR;
    const bool live = row < a.rows;   // a workgroup of several rows: the lanes of a row that is not there go along
    const uint64_t r = live ? row : a.rows - 1;
    const int at = (int)(threadIdx.x % TPR) * V, cols = (int)a.cols;
    const T *x = static_cast<const T *>(a.x) + r * a.x_stride;
    float v[CH][V];
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int j = at + c * TPR * V;
        const auto p = load_pack<T, V>(x + j, cols - j);
#pragma unroll
        for (int i = 0; i < V; ++i) { v[c][i] = (float)p[i]; s += v[c][i]; }
    }
    const float n = 1.0f / (float)cols;
    const float mean = row_sum<TPR>(s, lds) * n;
    s = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int j = at + c * TPR * V;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[c][i] = v[c][i] - mean;
            s += j + i < cols ? v[c][i] * v[c][i] : 0.f;
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum<TPR>(s, lds) * n + a.eps);
    if (!live) return;
    if (threadIdx.x % TPR == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int j = at + c * TPR * V;
        if (j >= cols) break;
        typename Pack<float, V>::V w, b;
#pragma unroll
        for (int i = 0; i < V; ++i) { w[i] = 1.f; b[i] = 0.f; }
        if (a.weight) w = load_pack<float, V>(a.weight + j, cols - j);
        if (a.bias) b = load_pack<float, V>(a.bias + j, cols - j);
        typename Pack<T, V>::V p;
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] = (T)(v[c][i] * rstd * w[i] + b[i]);
        store_pack<T, V>(y + j, cols - j, p);
    }
}

// Slices that a user's rows are cut into, one workgroup each.  A slice leaves a row of partial sums for either gradient, 16
// bytes a column written and read again, so it has 16 rows of three tensors.  Long rows, which a workgroup takes one at a time, are cut
// into slices of four while that leaves CUs without one (200 rows of 16000 bf16 elements, 13 or 50 slices: 75 or 37 us).
// However many there are, a slice's fp32 accumulators take 512 rows at most: 8192 terms of one sign have left a sum 1.2e-4 off.
constexpr uint32_t kMostTerms = 512;
static uint32_t backward_slices(uint32_t U, uint64_t rows, uint32_t cols)
{
    const auto slices = [&](uint64_t each, uint32_t in_all) {
        const uint64_t most = in_all / U > 1 ? in_all / U : 1, n = (rows + each - 1) / each;
        return (uint32_t)(n < 1 ? 1 : n < most ? n : most);
    };
    uint32_t n = slices(16, 512);
    if (cols > 1024 && n * U < 256) n = slices(4, 256);
    // rows of a workgroup at a time, each with accumulators of its own: of fp32 elements, and no fewer of 16 bits
    const uint32_t at_once = cols <= 32 ? 32 : cols <= 64 ? 16 : cols <= 128 ? 8 : cols <= 1024 ? 4 : 1;
    const uint64_t least = (rows + kMostTerms * at_once - 1) / (kMostTerms * at_once);
    return n < least ? (uint32_t)least : n;
}

// Where a slice's sums of a user go: to its place, or to the gradients themselves where it is the only one.
__device__ inline float *grad_place(const co3_layernorm_backward_args &a, uint32_t u, uint32_t slice, uint32_t slices, float *partial, bool bias)
{
    float *const grad = bias ? a.dbias : a.dweight;
    return slices > 1 ? partial + (((uint64_t)u * slices + slice) * 2 + (bias ? 1 : 0)) * a.cols : grad ? grad + u * a.grad_stride : nullptr;
}
template <int V>
__device__ inline void put_grad(float *to, int j, int cols, const float (&g)[V], bool add)
{
    if (!to) return;
    typename Pack<float, V>::V v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = g[i];
    if (add) v += load_pack<float, V>(to + j, cols - j);
    store_pack<float, V>(to + j, cols - j, v);
}

// GRADS: the weight's gradients too, in registers while the slice's rows go by.  At most two workgroups of 256 threads fit a CU with
// them (240 registers of 8192 bf16 columns), so xh and t are computed twice rather than kept: 249 us kept by workgroups of 512 threads, 209
// us with the next row asked for ahead instead, 175 us so.
template <typename T, int TPR, int CH, bool GRADS>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_layernorm_backward(co3_layernorm_backward_args a, uint32_t slices, float *partial)
{
    constexpr int V = kVec<T>, WG = TPR > 256 ? TPR : 256, ROWS = WG / TPR;
    __shared__ float lds[2][WG / 64][2];
    extern __shared__ float sums[];   // [2][cols], where several rows are on their way at a time
    const uint32_t u = blockIdx.y;
    const int sub = threadIdx.x / TPR, at = (int)(threadIdx.x % TPR) * V, cols = (int)a.cols;
    const uint64_t base = (uint64_t)u * a.rows_per_user;
    const uint64_t r0 = a.rows_per_user * blockIdx.x / slices, r1 = a.rows_per_user * (blockIdx.x + 1) / slices;
    const float n = 1.0f / (float)cols;
    float dw[CH][V], db[CH][V];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) dw[c][i] = db[c][i] = 0.f;
    constexpr bool kKeep = TPR <= 512;   // workgroups of 1024 threads have half the registers: they read the weights with every row
    typename Pack<float, V>::V w[kKeep ? CH : 1];
#pragma unroll
    for (int c = 0; c < (kKeep ? CH : 1); ++c) {
        const int j = at + c * TPR * V;
#pragma unroll
        for (int i = 0; i < V; ++i) w[c][i] = 1.f;
        if (a.weight && kKeep) w[c] = load_pack<float, V>(a.weight + j, cols - j);
    }
    for (uint64_t k = r0; k < r1; k += ROWS) {   // the same number of turns for all threads
        const bool live = k + sub < r1;
        const uint64_t r = base + (live ? k + sub : k);
        const T *x = static_cast<const T *>(a.x) + r * a.x_stride, *dy = static_cast<const T *>(a.dy) + r * a.dy_stride;
        typename Pack<T, V>::V px[CH], pd[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int j = at + c * TPR * V;
            px[c] = load_pack<T, V>(x + j, cols - j);
            pd[c] = load_pack<T, V>(dy + j, live ? cols - j : 0);   // a row that is not there adds nothing
        }
        const float mean = a.mean[r], rstd = a.rstd[r];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int j = at + c * TPR * V;
            typename Pack<float, V>::V wc = w[kKeep ? c : 0];
            if (a.weight && !kKeep) wc = load_pack<float, V>(a.weight + j, cols - j);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = (float)pd[c][i], t = d * wc[i];
                const float xh = live && j + i < cols ? ((float)px[c][i] - mean) * rstd : 0.f;
                s1 += t;
                s2 += t * xh;
                if (GRADS) dw[c][i] += d * xh;
                if (GRADS) db[c][i] += d;
            }
        }
        row_sums<TPR>(s1, s2, lds[(k - r0) / ROWS % 2]);
        s1 *= n;
        s2 *= n;
        if (!live) continue;
        T *dx = static_cast<T *>(a.dx) + r * a.dx_stride;
#pragma unroll
        for (int c = 0; c < CH; ++c) asm volatile("" : "+v"(px[c]), "+v"(pd[c]));   // xh and t are computed once more: no registers for them
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int j = at + c * TPR * V;
            if (j >= cols) break;
            typename Pack<T, V>::V p;
            typename Pack<float, V>::V wc = w[kKeep ? c : 0];
            if (a.weight && !kKeep) wc = load_pack<float, V>(a.weight + j, cols - j);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = ((float)px[c][i] - mean) * rstd;
                p[i] = (T)(rstd * ((float)pd[c][i] * wc[i] - s1 - xh * s2));
            }
            store_pack<T, V>(dx + j, cols - j, p);
        }
    }
    if (!GRADS || (!a.dweight && !a.dbias)) return;
    if (ROWS > 1) {   // the workgroup's rows after one another
        for (int w = 0; w < ROWS; ++w) {
            if (sub == w) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int j = at + c * TPR * V + i;
                        if (j >= cols) continue;
                        sums[j] = dw[c][i] = (w ? sums[j] : 0.f) + dw[c][i];
                        sums[cols + j] = db[c][i] = (w ? sums[cols + j] : 0.f) + db[c][i];
                    }
            }
            __syncthreads();
        }
        if (sub != ROWS - 1) return;
    }
    float *const to_w = grad_place(a, u, blockIdx.x, slices, partial, false), *const to_b = grad_place(a, u, blockIdx.x, slices, partial, true);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int j = at + c * TPR * V;
        put_grad<V>(to_w, j, cols, dw[c], slices == 1 && a.accumulate);
        put_grad<V>(to_b, j, cols, db[c], slices == 1 && a.accumulate);
    }
}

// The weight's gradients of rows that are too long for a workgroup's registers: a thread goes down a slice's rows in its columns.  x and dy
// are read twice then: 2000 x 32768 bf16 170 us, 395 us with gradients in registers that spill.
template <typename T>
__global__ __launch_bounds__(256) void k_layernorm_columns(co3_layernorm_backward_args a, uint32_t slices, float *partial)
{
    constexpr int V = kVec<T>;
    const uint32_t u = blockIdx.y;
    const int cols = (int)a.cols, j = (int)(blockIdx.z * 256 + threadIdx.x) * V;
    const uint64_t base = (uint64_t)u * a.rows_per_user;
    const uint64_t r0 = base + a.rows_per_user * blockIdx.x / slices, r1 = base + a.rows_per_user * (blockIdx.x + 1) / slices;
    float dw[V], db[V];
#pragma unroll
    for (int i = 0; i < V; ++i) dw[i] = db[i] = 0.f;
#pragma unroll 4
    for (uint64_t r = r0; r < r1; ++r) {
        const auto x = load_pack<T, V>(static_cast<const T *>(a.x) + r * a.x_stride + j, cols - j);
        const auto dy = load_pack<T, V>(static_cast<const T *>(a.dy) + r * a.dy_stride + j, cols - j);
        const float mean = a.mean[r], rstd = a.rstd[r];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            dw[i] += (float)dy[i] * (((float)x[i] - mean) * rstd);
            db[i] += (float)dy[i];
        }
    }
    put_grad<V>(grad_place(a, u, blockIdx.x, slices, partial, false), j, cols, dw, slices == 1 && a.accumulate);
    put_grad<V>(grad_place(a, u, blockIdx.x, slices, partial, true), j, cols, db, slices == 1 && a.accumulate);
}

// The slices' sums of a user, 64 columns of either gradient a workgroup: a wavefront takes every sixteenth slice.  In fp64, since there
// may be thousands of slices.
__global__ __launch_bounds__(1024) void k_layernorm_grad(co3_layernorm_backward_args a, uint32_t slices, const float *partial)
{
    __shared__ double part[16][64];
    const uint32_t u = blockIdx.y, lane = threadIdx.x & 63u, w = threadIdx.x >> 6;
    const uint64_t c = (uint64_t)blockIdx.x * 64 + lane, cols = a.cols;   // dweight's columns, then dbias's
    double s = 0.0;
    if (c < 2 * cols) {
        const float *p = partial + (uint64_t)u * slices * 2 * cols + c;
#pragma unroll 8
        for (uint32_t k = w; k < slices; k += 16) s += (double)p[k * 2 * cols];
    }
    part[w][lane] = s;
    __syncthreads();
    if (w || c >= 2 * cols) return;
    s = 0.0;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += part[k][lane];
    float *out = c < cols ? a.dweight : a.dbias;
    if (!out) return;
    out += u * a.grad_stride + (c < cols ? c : c - cols);
    *out = (float)(a.accumulate ? (double)*out + s : s);
}

// A launch of HIP has fewer than 2^32 threads: rows beyond that (2^22 by 1024 threads each, 2^29 by eight) have launches of their own.
template <typename T, int TPR, int CH>
static void forward(const co3_layernorm_args &a, hipStream_t s)
{
    constexpr int WG = TPR > 256 ? TPR : 256, ROWS = WG / TPR;
    constexpr uint64_t most = ((1ull << 32) - 1) / WG * ROWS;
    for (uint64_t row = 0; row < a.rows; row += most) {
        co3_layernorm_args part = a;
        part.rows = a.rows - row < most ? a.rows - row : most;
        part.x = static_cast<const T *>(a.x) + row * a.x_stride;
        part.y = static_cast<T *>(a.y) + row * a.y_stride;
        if (a.mean) part.mean = a.mean + row;
        if (a.rstd) part.rstd = a.rstd + row;
        k_layernorm<T, TPR, CH><<<dim3((uint32_t)((part.rows + ROWS - 1) / ROWS)), dim3(WG), 0, s>>>(part);
    }
}

template <typename T, int TPR, int CH>
static void backward(const co3_layernorm_backward_args &a, uint32_t slices, float *partial, hipStream_t s)
{
    constexpr int WG = TPR > 256 ? TPR : 256;
    if (TPR <= 512) {
        k_layernorm_backward<T, TPR, CH, TPR <= 512><<<dim3(slices, a.U), dim3(WG), WG > TPR ? 8 * a.cols : 0, s>>>(a, slices, partial);
        return;
    }
    if (a.dweight || a.dbias)   // first: dx may take the place of what they are made of
        k_layernorm_columns<T><<<dim3(slices, a.U, (a.cols + 256 * kVec<T> - 1) / (256 * kVec<T>)), dim3(256), 0, s>>>(a, slices, partial);
    const uint64_t most = a.U < 2048 ? 2048 / a.U : 1;
    const uint32_t rows = (uint32_t)(a.rows_per_user < most ? a.rows_per_user : most);
    if (rows) k_layernorm_backward<T, TPR, CH, TPR <= 512><<<dim3(rows, a.U), dim3(WG), 0, s>>>(a, rows, nullptr);
}

template <typename T> constexpr uint32_t kMostPacks = CO3_MAX_NORM_COLS / kVec<T>;   // of a row: 4096 of 16 bits, 8192 of fp32

template <typename T>
static void forward_of(const co3_layernorm_args &a, hipStream_t s)
{
    const uint32_t packs = (a.cols + kVec<T> - 1) / kVec<T>;
    if (packs <= 8) forward<T, 8, 1>(a, s);
    else if (packs <= 16) forward<T, 16, 1>(a, s);
    else if (packs <= 32) forward<T, 32, 1>(a, s);
    else if (packs <= 64) forward<T, 64, 1>(a, s);
    else if (packs <= 128) forward<T, 64, 2>(a, s);
    else if (packs <= 256) forward<T, 64, 4>(a, s);
    else if (packs <= 512) forward<T, 64, 8>(a, s);
    else if (packs <= 1024) forward<T, 256, 4>(a, s);
    else if (packs <= 2048) forward<T, 256, 8>(a, s);
    else if (packs <= 4096) forward<T, 1024, 4>(a, s);
    else if constexpr (kMostPacks<T> > 4096) forward<T, 1024, 8>(a, s);
}

template <typename T>
static void backward_of(const co3_layernorm_backward_args &a, uint32_t slices, float *partial, hipStream_t s)
{
    const uint32_t packs = (a.cols + kVec<T> - 1) / kVec<T>;
    if (packs <= 8) backward<T, 8, 1>(a, slices, partial, s);
    else if (packs <= 16) backward<T, 16, 1>(a, slices, partial, s);
    else if (packs <= 32) backward<T, 32, 1>(a, slices, partial, s);
    else if (packs <= 64) backward<T, 64, 1>(a, slices, partial, s);
    else if (packs <= 128) backward<T, 64, 2>(a, slices, partial, s);
    else if (packs <= 256) backward<T, 64, 4>(a, slices, partial, s);
    else if (packs <= 512) backward<T, 256, 2>(a, slices, partial, s);
    else if (packs <= 1024) backward<T, 256, 4>(a, slices, partial, s);
    else if (packs <= 2048) backward<T, 512, 4>(a, slices, partial, s);
    else if (packs <= 4096) backward<T, 1024, 4>(a, slices, partial, s);
    else if constexpr (kMostPacks<T> > 4096) backward<T, 1024, 8>(a, slices, partial, s);   // 128 registers, and 30 that spill
}

size_t layernorm_backward_workspace_bytes(uint32_t U, uint64_t rows_per_user, uint32_t cols)
{
    const uint32_t slices = backward_slices(U, rows_per_user, cols);
    return slices > 1 ? (size_t)U * slices * 2 * cols * sizeof(float) : 0;
}

hipError_t launch_layernorm(const co3_layernorm_args &a, hipStream_t s)
{
    ProfScope prof(K_LAYERNORM, s);
    if (a.type == CO3_F32) forward_of<float>(a, s);
    else if (a.type == CO3_BF16) forward_of<__bf16>(a, s);
    else forward_of<_Float16>(a, s);
    return hipGetLastError();
}

hipError_t launch_layernorm_backward(const co3_layernorm_backward_args &a, hipStream_t s)
{
    const bool grads = a.dweight || a.dbias;
    const uint32_t slices = backward_slices(a.U, a.rows_per_user, a.cols);
    float *partial = static_cast<float *>(a.workspace);
    {
        ProfScope prof(K_LAYERNORM_BACKWARD, s);
        if (a.type == CO3_F32) backward_of<float>(a, slices, partial, s);
        else if (a.type == CO3_BF16) backward_of<__bf16>(a, slices, partial, s);
        else backward_of<_Float16>(a, slices, partial, s);
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (grads && slices > 1) {
        ProfScope prof(K_LAYERNORM_GRAD, s);
        k_layernorm_grad<<<dim3((2 * a.cols + 63) / 64, a.U), dim3(1024), 0, s>>>(a, slices, partial);
    }
    return hipGetLastError();
}

}  // namespace co3
