// Newton-Schulz iteration of every matrix of a flat vector, and the update that Muon makes of it.
//
//   X_0 = G / (|G|_F + eps);   A = X X^T,  B = b A + c A A,  X <- a X + B X
//
// A launch does one product for all matrices, a workgroup one tile: tables made with the plan say which.  A and A A are
// symmetric: only tiles on and below the diagonal are computed, the others are written from them.  All three products
// take their operands as rows that are contiguous along the sum (X X^T, A A^T, B (X^T)^T), so X is kept with its transpose.
//
// Numbers.  The matrix instructions take fp16 and add in fp32.  X, A and B are held times 2^14, 2^14 and 2^13: X's singular
// values stay below 2 and B's below 7, so nothing overflows, and at 2^14 what matters is far from the smallest fp16 number
// (of 4096 x 25088 noise, X_0's entries are 1.6 on average).  Scales are powers of two: they round nothing.  X is a pair
// hi + lo of 22 bits, since small singular values grow up to a^steps times (485 at five steps of Muon's a = 3.4445)
// while large ones stay: the rounding of the iterate to 11 bits, spread over all directions, grows with them (a
// matrix of one dominant direction and 10^-3 noise: 9e-2 off, with the pair 2e-4).  Roundings of A and B need no pair for
// results of 16 bits: where the singular values are small, so are A and B beside a (2e-3 off, the size of bf16's own rounding).
#include "co3_internal.h"
#include "ortho.h"
#include "tensor_types.h"

namespace co3 {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr float kScaleX = 16384.f, kScaleB = 8192.f;   // 2^14, also of A; 2^13

struct Polynomial { float a, b, c; };

// ---- norm and layout ----------------------------------------------------------------------------------------

__device__ inline double block_sum(double v, double *lds)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}

// Partial sums of squares in fp64 (no fp32 input overflows or vanishes there).  With momentum: updates it first; its squares, or
// those of g + beta m, are what is summed.
template <typename T, bool MUON>
__global__ __launch_bounds__(256) void k_ortho_norm(OrthoLayout lay, OrthoCall c)
{
    __shared__ double lds[4];
    const PartDev part = lay.parts[blockIdx.x];
    const MatDev m = lay.mats[part.mat];
    constexpr int V = kVec<T>;
    double s = 0.0;
    for (uint32_t l = 0; l < part.lines; ++l) {
        const uint64_t at = m.offset + part.at + l * m.ld;
        for (uint64_t k = (uint64_t)threadIdx.x * V; k < part.len; k += 256 * V) {
            const int n = part.len - k < (uint64_t)V ? (int)(part.len - k) : V;
            const auto g = load_pack<T, V>(static_cast<const T *>(c.g) + at + k, n);
            if constexpr (MUON) {
                auto mo = load_pack<float, V>(c.momentum + at + k, n);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    mo[i] = c.beta * mo[i] + g[i];
                    const double u = c.nesterov ? g[i] + c.beta * mo[i] : mo[i];
                    s += u * u;
                }
                store_pack<float, V>(c.momentum + at + k, n, mo);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) s += (double)(float)g[i] * (double)(float)g[i];
            }
        }
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0) c.partial[blockIdx.x] = s;
}

__device__ inline void split(float v, _Float16 &hi, _Float16 &lo)
{
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// What a tile of 64 x 64 floats in LDS is read and written by: 65 words a row, so that neither eight columns of eight rows nor
// eight rows of eight columns meet in a bank.
constexpr int kPitch = 65;

// X_0 and its transpose, with the padding.
template <typename T, bool MUON, bool PAIR>
__global__ __launch_bounds__(256) void k_ortho_pack(OrthoLayout lay, OrthoCall c)
{
    __shared__ double lds[4];
    __shared__ float tile[kPackTile * kPitch];
    const TileDev t = lay.pack[blockIdx.x];
    const MatDev m = lay.mats[t.mat];
    double s = 0.0;
    for (uint32_t p = threadIdx.x; p < m.nparts; p += 256) s += c.partial[m.part + p];
    s = block_sum(s, lds);
    const bool finite = s < INFINITY;   // false for NaN too
    const double f = !finite ? (double)NAN : s > 0.0 ? (double)kScaleX / (sqrt(s) + (double)c.eps) : 0.0;
    if (!finite && t.i == 0 && t.j == 0 && threadIdx.x == 0 && c.status)
        atomicAdd(reinterpret_cast<unsigned long long *>(c.status + CO3_STAT_NONFINITE), 1ull);

    const uint32_t gr = (m.tall ? t.j : t.i) * kPackTile, gc = (m.tall ? t.i : t.j) * kPackTile;   // in the caller's matrix
    const uint32_t lane = threadIdx.x & 63u;
    for (uint32_t r = threadIdx.x >> 6; r < kPackTile; r += 4) {
        float v = 0.f;
        if (gr + r < m.rows && gc + lane < m.cols) {
            const uint64_t at = m.offset + (uint64_t)(gr + r) * m.ld + gc + lane;
            float u = (float)static_cast<const T *>(c.g)[at];
            if constexpr (MUON) u = c.nesterov ? u + c.beta * c.momentum[at] : c.momentum[at];
            v = (float)((double)u * f);
        }
        tile[r * kPitch + lane] = v;
    }
    __syncthreads();
    const uint64_t plane = (uint64_t)m.Mp * m.Np;
    _Float16 *x = c.planes + m.x, *xt = c.planes + m.xt;
#pragma unroll
    for (uint32_t pass = 0; pass < 4; ++pass) {
        const bool across = pass & 1u;                                  // the tile's columns
        const uint32_t r = (pass >> 1) * 32 + threadIdx.x / 8, k = threadIdx.x % 8 * 8;
        half8 hi, lo;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            _Float16 h, l;
            split(tile[across ? (k + i) * kPitch + r : r * kPitch + k + i], h, l);
            hi[i] = h;
            lo[i] = l;
        }
        if (across == (m.tall != 0)) {
            const uint64_t at = (uint64_t)(t.i * kPackTile + r) * m.Np + t.j * kPackTile + k;
            *reinterpret_cast<half8 *>(x + at) = hi;
            *reinterpret_cast<half8 *>(x + plane + at) = lo;
        } else {
            const uint64_t at = (uint64_t)(t.j * kPackTile + r) * m.Mp + t.i * kPackTile + k;
            *reinterpret_cast<half8 *>(xt + at) = hi;
            if (PAIR) *reinterpret_cast<half8 *>(xt + plane + at) = lo;
        }
    }
}

// ---- products -----------------------------------------------------------------------------------------------

enum { GRAM, SQUARE, PRODUCT, LAST };

// acc[i][j] += sum over k of P[i][k] Q[j][k] for a wavefront's 64 x 64 of a workgroup's 128 x 128, from rows of K elements.
constexpr int kDepth = 32, kRow = kDepth + 8;   // elements of a row in LDS; 16 bytes apart from the next
template <bool PAIR>
__device__ inline void multiply(const _Float16 *p, const _Float16 *q, uint64_t plane_p, uint64_t plane_q, uint32_t K, _Float16 *lds,
                                float16v (&acc)[2][2])
{
    constexpr int PL = PAIR ? 2 : 1, T = (int)kTile;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int wi = (w >> 1) * 64, wj = (w & 1) * 64;
    const int row = threadIdx.x >> 2, part = (threadIdx.x & 3) * 8;
    for (uint32_t k0 = 0; k0 < K; k0 += kDepth) {
        half8 v[2 * PL][2];
#pragma unroll
        for (int pl = 0; pl < 2 * PL; ++pl)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const _Float16 *src = pl < PL ? p + pl * plane_p : q + (pl - PL) * plane_q;
                v[pl][h] = *reinterpret_cast<const half8 *>(src + (uint64_t)(row + h * 64) * K + k0 + part);
            }
        __syncthreads();
#pragma unroll
        for (int pl = 0; pl < 2 * PL; ++pl)
#pragma unroll
            for (int h = 0; h < 2; ++h) *reinterpret_cast<half8 *>(lds + (pl * T + row + h * 64) * kRow + part) = v[pl][h];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kDepth; k += 16) {
            half8 a[PL][2], b[PL][2];
#pragma unroll
            for (int pl = 0; pl < PL; ++pl)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    a[pl][h] = *reinterpret_cast<const half8 *>(lds + (pl * T + wi + h * 32 + lane % 32) * kRow + k + lane / 32 * 8);
                    b[pl][h] = *reinterpret_cast<const half8 *>(lds + ((PL + pl) * T + wj + h * 32 + lane % 32) * kRow + k + lane / 32 * 8);
                }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (PAIR) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0][i], b[PL - 1][j], acc[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[PL - 1][i], b[0][j], acc[i][j], 0, 0, 0);
                    }
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0][i], b[0][j], acc[i][j], 0, 0, 0);
                }
        }
    }
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

// `turn`: which of the two transposes this step reads.
template <int OP, bool PAIR>
__global__ __launch_bounds__(256) void k_ortho_product(OrthoLayout lay, OrthoCall c, Polynomial f, uint32_t turn)
{
    constexpr int PL = PAIR ? 2 : 1;
    constexpr size_t kStage = sizeof(_Float16) * 2 * PL * kTile * kRow, kFold = sizeof(float) * 4 * 64 * kPitch;
    __shared__ __attribute__((aligned(16))) unsigned char lds[kStage > kFold ? kStage : kFold];
    const TileDev t = OP == GRAM || OP == SQUARE ? lay.gram[blockIdx.x] : lay.product[blockIdx.x];
    const MatDev &m = lay.mats[t.mat];
    const uint32_t K = OP == GRAM ? m.Np : m.Mp;
    const uint64_t plane_x = (uint64_t)m.Mp * m.Np, plane_a = (uint64_t)m.Mp * m.Mp;
    _Float16 *x = c.planes + m.x, *xt = c.planes + m.xt + turn * PL * plane_x, *xt_next = c.planes + m.xt + (turn ^ 1u) * PL * plane_x;
    _Float16 *a = c.planes + m.a, *b = c.planes + m.b;
    const _Float16 *p = OP == GRAM ? x : OP == SQUARE ? a : b;
    const _Float16 *q = OP == GRAM ? x : OP == SQUARE ? a : xt;

    float16v acc[2][2] = {};
    multiply<PAIR>(p + (uint64_t)t.i * kTile * K, q + (uint64_t)t.j * kTile * K, OP == GRAM ? plane_x : plane_a,
                   OP == SQUARE ? plane_a : plane_x, K, reinterpret_cast<_Float16 *>(lds), acc);
    __syncthreads();

    // A wavefront's 64 x 64 through LDS: along its rows first, then along its columns.
    const uint32_t lane = threadIdx.x & 63u, w = threadIdx.x >> 6;
    float *fold = reinterpret_cast<float *>(lds) + w * 64 * kPitch;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                fold[(i * 32 + e / 4 * 8 + lane / 32 * 4 + e % 4) * kPitch + j * 32 + lane % 32] = acc[i][j][e];
    __syncthreads();
    const uint32_t i0 = t.i * kTile + (w >> 1) * 64, j0 = t.j * kTile + (w & 1) * 64;
    const bool turned = OP == PRODUCT || (OP == LAST && m.tall) || ((OP == GRAM || OP == SQUARE) && t.i != t.j);
#pragma unroll
    for (uint32_t pass = 0; pass < 8; ++pass) {
        const uint32_t r = pass * 8 + lane / 8, k = lane % 8 * 8;
        float *at = fold + r * kPitch + k;
        const uint64_t to = (uint64_t)(i0 + r) * (OP == PRODUCT || OP == LAST ? m.Np : m.Mp) + j0 + k;
        float v[8];
        half8 hi, lo;
        if (OP == SQUARE || OP == PRODUCT || OP == LAST) {
            const _Float16 *old = OP == SQUARE ? a : x;
            hi = *reinterpret_cast<const half8 *>(old + to);
            lo = half8{};
            if (PAIR || OP != SQUARE) lo = *reinterpret_cast<const half8 *>(old + (OP == SQUARE ? plane_a : plane_x) + to);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (OP == GRAM) v[e] = at[e] * (1.f / kScaleX);
            if (OP == SQUARE) v[e] = ((float)hi[e] + (float)lo[e]) * (f.b * (kScaleB / kScaleX)) + at[e] * (f.c * (kScaleB / kScaleX / kScaleX));
            if (OP == PRODUCT || OP == LAST) v[e] = f.a * ((float)hi[e] + (float)lo[e]) + at[e] * (1.f / kScaleB);
        }
        if (OP == LAST) {
            if (!m.tall) store_result(lay, c, m, i0 + r, j0 + k, v);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) at[e] = v[e];
            continue;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            _Float16 h, l;
            split(v[e], h, l);
            hi[e] = h;
            lo[e] = l;
            const uint32_t both = (uint32_t)__builtin_bit_cast(uint16_t, h) | (uint32_t)__builtin_bit_cast(uint16_t, l) << 16;
            at[e] = __builtin_bit_cast(float, both);
        }
        _Float16 *dst = OP == GRAM ? a : OP == SQUARE ? b : x;
        *reinterpret_cast<half8 *>(dst + to) = hi;
        if (PAIR || OP == PRODUCT) *reinterpret_cast<half8 *>(dst + (OP == PRODUCT ? plane_x : plane_a) + to) = lo;
    }
    if (!turned) return;   // the same for the whole workgroup
    __syncthreads();
#pragma unroll
    for (uint32_t pass = 0; pass < 8; ++pass) {
        const uint32_t r = pass * 8 + lane / 8, k = lane % 8 * 8;   // column r of the tile, rows k ..
        if (OP == LAST) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fold[(k + e) * kPitch + r];
            store_result(lay, c, m, j0 + r, i0 + k, v);
            continue;
        }
        half8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t both = __builtin_bit_cast(uint32_t, fold[(k + e) * kPitch + r]);
            hi[e] = __builtin_bit_cast(_Float16, (uint16_t)both);
            lo[e] = __builtin_bit_cast(_Float16, (uint16_t)(both >> 16));
        }
        _Float16 *dst = OP == GRAM ? a : OP == SQUARE ? b : xt_next;
        const uint64_t to = (uint64_t)(j0 + r) * m.Mp + i0 + k;
        *reinterpret_cast<half8 *>(dst + to) = hi;
        if (PAIR) *reinterpret_cast<half8 *>(dst + (OP == PRODUCT ? plane_x : plane_a) + to) = lo;
    }
}

// ---- the call -----------------------------------------------------------------------------------------------

template <typename T, bool MUON, bool PAIR>
static hipError_t iterate(const OrthoLayout &lay, const OrthoCall &c, hipStream_t s)
{
    {
        ProfScope prof(K_ORTHO_NORM, s);
        k_ortho_norm<T, MUON><<<dim3(lay.nparts), dim3(256), 0, s>>>(lay, c);
    }
    {
        ProfScope prof(K_ORTHO_PACK, s);
        k_ortho_pack<T, MUON, PAIR><<<dim3(lay.npack), dim3(256), 0, s>>>(lay, c);
    }
    for (uint32_t k = 0; k < c.steps; ++k) {
        const Polynomial f = {c.coefficients[3 * k], c.coefficients[3 * k + 1], c.coefficients[3 * k + 2]};
        {
            ProfScope prof(K_ORTHO_GRAM, s);
            k_ortho_product<GRAM, PAIR><<<dim3(lay.ngram), dim3(256), 0, s>>>(lay, c, f, 0);
        }
        {
            ProfScope prof(K_ORTHO_SQUARE, s);
            k_ortho_product<SQUARE, PAIR><<<dim3(lay.ngram), dim3(256), 0, s>>>(lay, c, f, 0);
        }
        ProfScope prof(K_ORTHO_PRODUCT, s);
        if (k + 1 < c.steps) k_ortho_product<PRODUCT, PAIR><<<dim3(lay.nproduct), dim3(256), 0, s>>>(lay, c, f, k & 1u);
        else k_ortho_product<LAST, PAIR><<<dim3(lay.nproduct), dim3(256), 0, s>>>(lay, c, f, k & 1u);
    }
    return hipGetLastError();
}

template <bool PAIR>
static hipError_t iterate_of(const OrthoLayout &lay, const OrthoCall &c, hipStream_t s)
{
    if (!c.out) return iterate<float, true, PAIR>(lay, c, s);
    if (lay.type == CO3_F32) return iterate<float, false, PAIR>(lay, c, s);
    if (lay.type == CO3_BF16) return iterate<__bf16, false, PAIR>(lay, c, s);
    return iterate<_Float16, false, PAIR>(lay, c, s);
}

hipError_t launch_orthogonalize(const OrthoLayout &lay, const OrthoCall &c, hipStream_t s)
{
    return lay.products == CO3_PRODUCTS_PAIR ? iterate_of<true>(lay, c, s) : iterate_of<false>(lay, c, s);
}

}  // namespace co3
