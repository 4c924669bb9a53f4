// Newton-Schulz iteration of matrices of up to 64 x 128: a workgroup takes one through all steps, in LDS and registers, in one launch.
//
// The same steps, scales and diagonals as in k_ortho.hip, which says what they are.  X stays in registers in fp32, as the matrix
// instructions leave it: a wavefront has 32 x 32 of it, a lane one column and four rows at a time.  Pairs hi + lo of X, X^T, A and B
// (or hi alone) are in LDS, whose rows are 8 numbers longer than they need: the same 16 bytes of sixteen rows lie in different banks.
// A and B are symmetric: a lane's four rows of a column are written as four columns of a row.
//
// Bound by the chain of its phases: three products a step, each with LDS reads, some hundred vector instructions a wavefront and a
// meeting of the workgroup behind it.  64 x 64 from high parts 1.8 us a step, 64 x 128 in pairs 3.6 us, and 8 us for the launch, the norm
// and the ends (the seventeen launches of k_ortho.hip: 70 to 80 us).
#include "co3_internal.h"
#include "ortho_device.h"

namespace co3 {

namespace {

typedef _Float16 half4 __attribute__((ext_vector_type(4)));
// X times 2^7, so that A comes out times 2^14; B times 2^13.
constexpr float kX7 = 128.f, kInvA = 1.f / kScaleX, kInvB = 1.f / kScaleB;
constexpr int kWaves = 8, kX = kSmallN + 8, kA = kSmallM + 8, kFlat = kSmallN + 1;   // elements between rows

struct Planes {
    _Float16 x[2][kSmallM * kX], xt[2][kSmallN * kA], a[2][kSmallM * kA], b[2][kSmallM * kA];
    float flat[kSmallM * kFlat];          // X row by row, on its way in and out
    float diag_a[kSmallM], diag_b[kSmallM];
    double sums[kWaves];
};

// acc (+)= P Q^T over up to 64 columns from k on, and to `end` at most, of 32 rows of each; `small` gets the products with low parts.
template <bool PAIR, bool FIRST>
__device__ inline void multiply(const _Float16 *p_hi, const _Float16 *p_lo, const _Float16 *q_hi, const _Float16 *q_lo, int ld_p, int ld_q,
                                int k, int end, float16v &acc, float16v (&small)[2])
{
    constexpr int n = 4;
    const int lane = threadIdx.x & 63, at_p = lane % 32 * ld_p + lane / 32 * 8, at_q = lane % 32 * ld_q + lane / 32 * 8;
    half8 ph[n], pl[n], qh[n], ql[n];
#pragma unroll
    for (int i = 0; i < n; ++i) {
        const int at = k + i * 16;   // behind the end too, unused: rows are as long
        ph[i] = *reinterpret_cast<const half8 *>(p_hi + at_p + at);
        qh[i] = *reinterpret_cast<const half8 *>(q_hi + at_q + at);
        if (PAIR) {
            pl[i] = *reinterpret_cast<const half8 *>(p_lo + at_p + at);
            ql[i] = *reinterpret_cast<const half8 *>(q_lo + at_q + at);
        }
    }
#pragma unroll
    for (int i = 0; i < n; ++i) {   // sums in turn, none of which waits for itself
        if (i && k + i * 16 >= end) break;
        const bool none = FIRST && i == 0;
        if (PAIR) small[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[i], ql[i], none ? float16v{} : small[0], 0, 0, 0);
        if (PAIR) small[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl[i], qh[i], none ? float16v{} : small[1], 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[i], qh[i], none ? float16v{} : acc, 0, 0, 0);
    }
}
template <bool PAIR>
__device__ inline float total(const float16v &acc, const float16v (&small)[2], int e)
{
    return PAIR ? acc[e] + (small[0][e] + small[1][e]) : acc[e];
}

template <bool PAIR>
__device__ inline void put4(_Float16 *hi, _Float16 *lo, const float (&v)[4])
{
    half4 h, l;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        _Float16 a, b;
        split(v[i], a, b);
        h[i] = a;
        l[i] = b;
    }
    *reinterpret_cast<half4 *>(hi) = h;
    if (PAIR) *reinterpret_cast<half4 *>(lo) = l;
}

}  // namespace

template <typename T, bool MUON, bool PAIR>
__global__ __launch_bounds__(64 * kWaves) void k_ortho_small(OrthoLayout lay, OrthoCall c)
{
    __shared__ __attribute__((aligned(16))) Planes s;
    const MatDev m = lay.mats[blockIdx.x];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, w = tid >> 6, col = lane % 32, row = lane / 32 * 4;

    // The matrix as it lies, line by line: X's rows, or its columns.
    const uint32_t line = m.tall ? kSmallM : kSmallN, per = 64 * kWaves / line, k = tid % line, first = tid / line;
    constexpr int kEach = kSmallM * kSmallN / (64 * kWaves);
    double squares = 0.0;
    {
        uint64_t at[kEach];
        float u[kEach], mo[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {   // all at once: elements that are not there are the matrix's last ones, unused
            const uint32_t r = first + i * per;
            at[i] = m.offset + (uint64_t)(r < m.rows ? r : m.rows - 1) * m.ld + (k < m.cols ? k : m.cols - 1);
            u[i] = (float)static_cast<const T *>(c.g)[at[i]];
            if constexpr (MUON) mo[i] = c.momentum[at[i]];
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t r = first + i * per;
            const bool there = r < m.rows && k < m.cols;
            if constexpr (MUON) {
                mo[i] = c.beta * mo[i] + u[i];
                u[i] = c.nesterov ? u[i] + c.beta * mo[i] : mo[i];
            }
            u[i] = there ? u[i] : 0.f;
            squares += (double)u[i] * (double)u[i];
            s.flat[m.tall ? k * kFlat + r : r * kFlat + k] = u[i];
        }
        if constexpr (MUON) {
            __syncthreads();   // all have read theirs
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (first + i * per < m.rows && k < m.cols) c.momentum[at[i]] = mo[i];
        }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) squares += __shfl_xor(squares, o);
    if (lane == 0) s.sums[w] = squares;
    __syncthreads();
    squares = 0.0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) squares += s.sums[i];
    const double scale = scale_of(squares, c.eps) * (double)(kX7 / kScaleX);
    if (scale != scale && tid == 0) count_not_finite(c);

    // The wavefront's 32 x 32 of X, and the first four's of A and B; what lies outside the matrix is neither written nor read.
    const uint32_t xi = w % 2 * 32, xj = w / 2 * 32, ai = w % 4 / 2 * 32, aj = w % 2 * 32;
    const bool has_x = xi < m.M && xj < m.N, has_a = w < 4 && ai < m.M && aj < m.M;
    float x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = (float)((double)s.flat[(xi + e / 4 * 8 + row + e % 4) * kFlat + xj + col] * scale);

    for (uint32_t step = 0; step < c.steps; ++step) {
        const float fa = c.coefficients[3 * step], fb = c.coefficients[3 * step + 1], fc = c.coefficients[3 * step + 2];
        float16v acc, small[2];
        if (has_x) {   // X and X^T; all have read the former ones
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const uint32_t r = xi + e / 4 * 8 + row, n = xj + col;
                const float v[4] = {x[e], x[e + 1], x[e + 2], x[e + 3]};
                put4<PAIR>(&s.xt[0][n * kA + r], &s.xt[1][n * kA + r], v);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    _Float16 h, l;
                    split(v[i], h, l);
                    s.x[0][(r + i) * kX + n] = h;
                    if (PAIR) s.x[1][(r + i) * kX + n] = l;
                }
            }
        }
        __syncthreads();
        // A
        if (has_a) {
            const _Float16 *ph = s.x[0] + ai * kX, *pl = s.x[1] + ai * kX, *qh = s.x[0] + aj * kX, *ql = s.x[1] + aj * kX;
            multiply<PAIR, true>(ph, pl, qh, ql, kX, kX, 0, (int)m.N, acc, small);
            if (m.N > 64) multiply<PAIR, false>(ph, pl, qh, ql, kX, kX, 64, (int)m.N, acc, small);
            float d = 0.f;
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const uint32_t r = ai + e / 4 * 8 + row, n = aj + col;
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = total<PAIR>(acc, small, e + i);
                    if (ai == aj) {   // the diagonal's tiles
                        d = r + i == n ? v[i] : d;
                        v[i] = r + i == n ? 0.f : v[i];
                    }
                }
                put4<PAIR>(&s.a[0][n * kA + r], &s.a[1][n * kA + r], v);
            }
            if (ai == aj && (col / 4 & 1) == row / 4) s.diag_a[aj + col] = d;   // the lane that has the column's element
        }
        __syncthreads();
        // B
        if (has_a) {
            multiply<PAIR, true>(s.a[0] + ai * kA, s.a[1] + ai * kA, s.a[0] + aj * kA, s.a[1] + aj * kA, kA, kA, 0, (int)m.M, acc, small);
            const float dn = s.diag_a[aj + col], base = fmaf(dn, fc * kInvA * 0.5f, fb * 0.5f), cc = fc * kInvA * 0.5f;
            float d_b = 0.f;
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const uint32_t r = ai + e / 4 * 8 + row, n = aj + col;
                const half4 h = *reinterpret_cast<const half4 *>(&s.a[0][n * kA + r]);
                half4 l = {};
                if (PAIR) l = *reinterpret_cast<const half4 *>(&s.a[1][n * kA + r]);
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {   // half of B times 2^14
                    float a = (float)h[i] + (float)l[i], t = fmaf(s.diag_a[r + i], cc, base);
                    if (ai == aj) {
                        a = r + i == n ? dn : a;
                        t = r + i == n ? base : t;
                    }
                    v[i] = fmaf(t, a, cc * total<PAIR>(acc, small, e + i));
                    if (ai == aj) {
                        d_b = r + i == n ? v[i] : d_b;
                        v[i] = r + i == n ? 0.f : v[i];
                    }
                }
                put4<PAIR>(&s.b[0][n * kA + r], &s.b[1][n * kA + r], v);
            }
            if (ai == aj && (col / 4 & 1) == row / 4) s.diag_b[aj + col] = d_b;
        }
        __syncthreads();
        // X
        if (has_x) {
            multiply<PAIR, true>(s.b[0] + xi * kA, s.b[1] + xi * kA, s.xt[0] + xj * kA, s.xt[1] + xj * kA, kA, kA, 0, (int)m.M, acc, small);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float d = s.diag_b[xi + e / 4 * 8 + row + e % 4];
                const float kept = PAIR ? x[e] * fmaf(d, kInvB, fa) : fmaf(x[e], fa, (float)(_Float16)x[e] * (d * kInvB));
                x[e] = fmaf(total<PAIR>(acc, small, e), kInvB, kept);
            }
        }
        __syncthreads();
    }

#pragma unroll
    for (int e = 0; e < 16; ++e) s.flat[(xi + e / 4 * 8 + row + e % 4) * kFlat + xj + col] = x[e];
    __syncthreads();
    const float out_scale = m.scale / kX7, keep = 1.f - c.eta * c.decay;
#pragma unroll 8
    for (int i = 0; i < kEach; ++i) {
        const uint32_t r = first + i * per;
        if (r >= m.rows || k >= m.cols) continue;
        const uint64_t at = m.offset + (uint64_t)r * m.ld + k;
        const float v = s.flat[m.tall ? k * kFlat + r : r * kFlat + k];
        if constexpr (MUON) c.model[at] = c.model[at] * keep - c.eta * out_scale * v;
        else static_cast<T *>(c.out)[at] = (T)(v * out_scale);
    }
}

template <bool PAIR>
static void small(const OrthoLayout &lay, const OrthoCall &c, hipStream_t s)
{
    const dim3 grid(lay.nmat), block(64 * kWaves);
    if (!c.out) k_ortho_small<float, true, PAIR><<<grid, block, 0, s>>>(lay, c);
    else if (lay.type == CO3_F32) k_ortho_small<float, false, PAIR><<<grid, block, 0, s>>>(lay, c);
    else if (lay.type == CO3_BF16) k_ortho_small<__bf16, false, PAIR><<<grid, block, 0, s>>>(lay, c);
    else k_ortho_small<_Float16, false, PAIR><<<grid, block, 0, s>>>(lay, c);
}

hipError_t launch_orthogonalize_small(const OrthoLayout &lay, const OrthoCall &c, hipStream_t s)
{
    ProfScope prof(K_ORTHO_SMALL, s);
    if (lay.products == CO3_PRODUCTS_PAIR) small<true>(lay, c, s);
    else small<false>(lay, c, s);
    return hipGetLastError();
}

}  // namespace co3
