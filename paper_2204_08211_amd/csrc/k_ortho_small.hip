// Newton-Schulz iteration of matrices of up to 64 x 128: a workgroup takes one through all steps, in LDS and registers, in one launch.
//
// The same steps, scales and diagonals as in k_ortho.hip, which says what they are.  X stays in registers in fp32, as the matrix
// instructions leave it: a wavefront has 32 x 32 of it, a lane one column and four rows at a time.  Pairs hi + lo of X, X^T, A and B
// (or hi alone) are in LDS, whose rows are 8 numbers longer than they need: the same 16 bytes of sixteen rows lie in different banks.
// A and B are symmetric: a lane's four rows of a column are written as four columns of a row.
//
// Bound by the chain of its phases: three products a step, each with LDS reads, some hundred vector instructions a wavefront and a
// meeting of the workgroup behind it.  64 x 64 in pairs 2.4 us a step (from high parts 1.8), 64 x 128 3.6 us, and 8 us for the launch, the norm
// and the ends (the seventeen launches of k_ortho.hip: 70 to 80 us).
//
// Matrices of as few rows and more columns (k_ortho_thin): a workgroup has 128 columns, a launch is a step.  Five steps of 64 x 1024 fp32
// 56 us, of 64 x 8192 98 us, of 2 x 777 42 us (by the products' launches 117, 147 and 114 us): bound by the chain of a launch, its first loads
// and the phases, 6 us, and 0.15 us for every part of A that is added up.
#include "co3_internal.h"
#include "ortho_device.h"

namespace co3 {

namespace {

typedef _Float16 half4 __attribute__((ext_vector_type(4)));
// X times 2^7, so that A comes out times 2^14; B times 2^13.
constexpr float kX7 = 128.f, kX10 = 1024.f, kInvA = 1.f / kScaleX, kInvB = 1.f / kScaleB;
constexpr int kWaves = 8, kX = kSmallN + 8, kA = kSmallM + 8, kFlat = kSmallN + 1;   // elements between rows
constexpr int kEach = kSmallM * kSmallN / (64 * kWaves);

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

// What a thread has: its wavefront's 32 x 32 of X from xi, xj on, and the first four wavefronts' of A and B from ai, aj on; of these,
// column `col` and four rows from `row` on at a time.  What lies outside the matrix is neither written nor read.
struct Part {
    uint32_t xi, xj, ai, aj, row, col;
    bool has_x, has_a;
};
__device__ inline Part part_of(uint32_t M, uint32_t N)
{
    const uint32_t lane = threadIdx.x & 63u, w = threadIdx.x >> 6;
    Part p = {w % 2 * 32, w / 2 * 32, w % 4 / 2 * 32, w % 2 * 32, lane / 32 * 4, lane % 32, false, false};
    p.has_x = p.xi < M && p.xj < N;
    p.has_a = w < 4 && p.ai < M && p.aj < M;
    return p;
}

// X^T
template <bool PAIR>
__device__ inline void put_columns(Planes &s, const Part &p, const float (&x)[16])
{
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        const uint32_t r = p.xi + e / 4 * 8 + p.row, n = p.xj + p.col;
        const float v[4] = {x[e], x[e + 1], x[e + 2], x[e + 3]};
        put4<PAIR>(&s.xt[0][n * kA + r], &s.xt[1][n * kA + r], v);
    }
}
// X
template <bool PAIR>
__device__ inline void put_rows(Planes &s, const Part &p, const float (&x)[16])
{
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const uint32_t r = p.xi + e / 4 * 8 + p.row + e % 4, n = p.xj + p.col;
        _Float16 h, l;
        split(x[e], h, l);
        s.x[0][r * kX + n] = h;
        if (PAIR) s.x[1][r * kX + n] = l;
    }
}
// X X^T
template <bool PAIR>
__device__ inline void gram(const Planes &s, const Part &p, uint32_t N, float (&v)[16])
{
    const _Float16 *ph = s.x[0] + p.ai * kX, *pl = s.x[1] + p.ai * kX, *qh = s.x[0] + p.aj * kX, *ql = s.x[1] + p.aj * kX;
    float16v acc, small[2];
    multiply<PAIR, true>(ph, pl, qh, ql, kX, kX, 0, (int)N, acc, small);
    if (N > 64) multiply<PAIR, false>(ph, pl, qh, ql, kX, kX, 64, (int)N, acc, small);
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = total<PAIR>(acc, small, e);
}
// A of its values, and its diagonal
template <bool PAIR>
__device__ inline void put_a(Planes &s, const Part &p, const float (&a)[16])
{
    float d = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        const uint32_t r = p.ai + e / 4 * 8 + p.row, n = p.aj + p.col;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = a[e + i];
            if (p.ai == p.aj) {   // the diagonal's tiles
                d = r + i == n ? v[i] : d;
                v[i] = r + i == n ? 0.f : v[i];
            }
        }
        put4<PAIR>(&s.a[0][n * kA + r], &s.a[1][n * kA + r], v);
    }
    if (p.ai == p.aj && (p.col / 4 & 1) == p.row / 4) s.diag_a[p.aj + p.col] = d;   // the lane that has the column's element
}
// B
template <bool PAIR>
__device__ inline void make_b(Planes &s, const Part &p, uint32_t M, float fb, float fc)
{
    float16v acc, small[2];
    multiply<PAIR, true>(s.a[0] + p.ai * kA, s.a[1] + p.ai * kA, s.a[0] + p.aj * kA, s.a[1] + p.aj * kA, kA, kA, 0, (int)M, acc, small);
    const float dn = s.diag_a[p.aj + p.col], base = fmaf(dn, fc * kInvA * 0.5f, fb * 0.5f), cc = fc * kInvA * 0.5f;
    float d_b = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        const uint32_t r = p.ai + e / 4 * 8 + p.row, n = p.aj + p.col;
        const half4 h = *reinterpret_cast<const half4 *>(&s.a[0][n * kA + r]);
        half4 l = {};
        if (PAIR) l = *reinterpret_cast<const half4 *>(&s.a[1][n * kA + r]);
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // half of B times 2^14
            float a = (float)h[i] + (float)l[i], t = fmaf(s.diag_a[r + i], cc, base);
            if (p.ai == p.aj) {
                a = r + i == n ? dn : a;
                t = r + i == n ? base : t;
            }
            v[i] = fmaf(t, a, cc * total<PAIR>(acc, small, e + i));
            if (p.ai == p.aj) {
                d_b = r + i == n ? v[i] : d_b;
                v[i] = r + i == n ? 0.f : v[i];
            }
        }
        put4<PAIR>(&s.b[0][n * kA + r], &s.b[1][n * kA + r], v);
    }
    if (p.ai == p.aj && (p.col / 4 & 1) == p.row / 4) s.diag_b[p.aj + p.col] = d_b;
}
// a X + B X
template <bool PAIR>
__device__ inline void update(const Planes &s, const Part &p, uint32_t M, float fa, float (&x)[16])
{
    float16v acc, small[2];
    multiply<PAIR, true>(s.b[0] + p.xi * kA, s.b[1] + p.xi * kA, s.xt[0] + p.xj * kA, s.xt[1] + p.xj * kA, kA, kA, 0, (int)M, acc, small);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const float d = s.diag_b[p.xi + e / 4 * 8 + p.row + e % 4];
        const float kept = PAIR ? x[e] * fmaf(d, kInvB, fa) : fmaf(x[e], fa, (float)(_Float16)x[e] * (d * kInvB));
        x[e] = fmaf(total<PAIR>(acc, small, e), kInvB, kept);
    }
}
__device__ inline double all_sums(double v, double *lds)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63u) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) v += lds[i];
    return v;
}
// `rows` by `cols` of the caller's matrix, from `base` on, are X's result: of it, or of its transpose where it is tall.
template <typename T, bool MUON>
__device__ inline void put_result(const OrthoCall &c, const MatDev &m, const float *flat, uint64_t base, uint32_t rows, uint32_t cols,
                                  float scale)
{
    const uint32_t line = m.tall ? kSmallM : kSmallN, per = 64 * kWaves / line, k = threadIdx.x % line, first = threadIdx.x / line;
    const float keep = 1.f - c.eta * c.decay;
#pragma unroll 8
    for (int i = 0; i < kEach; ++i) {
        const uint32_t r = first + i * per;
        if (r >= rows || k >= cols) continue;
        const uint64_t at = base + (uint64_t)r * m.ld + k;
        const float v = flat[m.tall ? k * kFlat + r : r * kFlat + k];
        if constexpr (MUON) c.model[at] = c.model[at] * keep - c.eta * scale * v;
        else static_cast<T *>(c.out)[at] = (T)(v * scale);
    }
}

}  // namespace

template <typename T, bool MUON, bool PAIR>
__global__ __launch_bounds__(64 * kWaves) void k_ortho_small(OrthoLayout lay, OrthoCall c)
{
    __shared__ __attribute__((aligned(16))) Planes s;
    const MatDev m = lay.mats[blockIdx.x];
    const uint32_t tid = threadIdx.x;

    // The matrix as it lies, line by line: X's rows, or its columns.
    const uint32_t line = m.tall ? kSmallM : kSmallN, per = 64 * kWaves / line, k = tid % line, first = tid / line;
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
    squares = all_sums(squares, s.sums);
    const double scale = scale_of(squares, c.eps) * (double)(kX7 / kScaleX);
    if (scale != scale && tid == 0) count_not_finite(c);

    const Part p = part_of(m.M, m.N);
    float x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = (float)((double)s.flat[(p.xi + e / 4 * 8 + p.row + e % 4) * kFlat + p.xj + p.col] * scale);

    for (uint32_t step = 0; step < c.steps; ++step) {
        if (p.has_x) {   // all have read the former ones
            put_columns<PAIR>(s, p, x);
            put_rows<PAIR>(s, p, x);
        }
        __syncthreads();
        if (p.has_a) {
            float a[16];
            gram<PAIR>(s, p, m.N, a);
            put_a<PAIR>(s, p, a);
        }
        __syncthreads();
        if (p.has_a) make_b<PAIR>(s, p, m.M, c.coefficients[3 * step + 1], c.coefficients[3 * step + 2]);
        __syncthreads();
        if (p.has_x) update<PAIR>(s, p, m.M, c.coefficients[3 * step], x);
        __syncthreads();
    }

#pragma unroll
    for (int e = 0; e < 16; ++e) s.flat[(p.xi + e / 4 * 8 + p.row + e % 4) * kFlat + p.xj + p.col] = x[e];
    __syncthreads();
    put_result<T, MUON>(c, m, s.flat, m.offset, m.rows, m.cols, m.scale / kX7);
}

// The same for matrices of up to 64 rows and any number of columns (their transposes'): a workgroup has 128 columns of X and a launch takes
// the step's B from A, X from B, and leaves the columns' part of the next A.  Launch 0 lays X out, the last one writes the result.  A's
// parts, of 32 x 32 or 64 x 64, are added up by every workgroup in the same order; they lie in two places, which launches take in turn.
// X times 2^10: entries of long rows are small.
template <typename T, bool MUON, bool PAIR>
__global__ __launch_bounds__(64 * kWaves) void k_ortho_thin(OrthoLayout lay, OrthoCall c, Polynomial f, uint32_t step)
{
    typedef float float4v __attribute__((ext_vector_type(4)));
    __shared__ __attribute__((aligned(16))) Planes s;
    const TileDev t = lay.pack.tiles[blockIdx.x];
    const MatDev m = lay.mats[t.mat];
    const uint32_t tid = threadIdx.x, strips = (m.N + kSmallN - 1) / kSmallN, side = m.M > 32 ? 64u : 32u;
    const uint32_t n0 = t.j * kSmallN, n = m.N - n0 < kSmallN ? m.N - n0 : kSmallN;
    const uint32_t rows = m.tall ? n : m.M, cols = m.tall ? m.M : n;      // the caller's, of this strip, from `base` on
    const uint64_t base = m.offset + (m.tall ? (uint64_t)n0 * m.ld : n0), part = side * side;
    float *const grams = c.sums + m.a;
    float4v *const kept = reinterpret_cast<float4v *>(c.sums + m.x) + (uint64_t)t.j * 4 * 64 * kWaves + tid;
    const Part p = part_of(m.M, n);
    float x[16];
    if (step == 0) {
        double squares = 0.0;
        for (uint32_t q = tid; q < m.nparts; q += 64 * kWaves) squares += c.partial[m.part + q];
        squares = all_sums(squares, s.sums);
        const double scale = scale_of(squares, c.eps) * (double)(kX10 / kScaleX);
        if (scale != scale && t.j == 0 && tid == 0) count_not_finite(c);
        const uint32_t line = m.tall ? kSmallM : kSmallN, per = 64 * kWaves / line, k = tid % line, first = tid / line;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const uint32_t r = first + i * per;
            const uint64_t at = base + (uint64_t)(r < rows ? r : rows - 1) * m.ld + (k < cols ? k : cols - 1);
            float u = (float)static_cast<const T *>(c.g)[at];
            if constexpr (MUON) u = c.nesterov ? u + c.beta * c.momentum[at] : c.momentum[at];
            s.flat[m.tall ? k * kFlat + r : r * kFlat + k] = r < rows && k < cols ? u : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = (float)((double)s.flat[(p.xi + e / 4 * 8 + p.row + e % 4) * kFlat + p.xj + p.col] * scale);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4v v = p.has_x ? kept[i * 64 * kWaves] : float4v{};
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * i + e] = v[e];
        }
        // Four elements a place.  64 x 64: a thread adds two places up; 32 x 32: every fourth part of one, twice.
        const bool wide = side == 64;
        const float4v *from = reinterpret_cast<const float4v *>(grams + ((step - 1) & 1u) * strips * part);
        const uint32_t at0 = wide ? tid : tid % 256, at1 = wide ? tid + 512 : at0, by = wide ? 1u : 4u;
        const uint32_t q0 = wide ? 0u : tid / 256, q1 = wide ? 0u : q0 + 2;
        float4v sum0 = {}, sum1 = {};
#pragma unroll 8
        for (uint32_t q = 0; q < strips; q += by) {
            const uint32_t a = q + q0 < strips ? q + q0 : strips - 1, b = q + q1 < strips ? q + q1 : strips - 1;
            const float4v va = from[a * (part / 4) + at0], vb = from[b * (part / 4) + at1];
            sum0 += q + q0 < strips ? va : float4v{};
            sum1 += q + q1 < strips ? vb : float4v{};
        }
        if (!wide) sum0 += sum1;
        const uint32_t to = wide ? at0 / 16 * kFlat + at0 % 16 * 4 : (at0 / 8 + tid / 256 * 32) * kFlat + at0 % 8 * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s.flat[to + i] = sum0[i];
            if (wide) s.flat[to + 32 * kFlat + i] = sum1[i];
        }
        if (p.has_x) put_columns<PAIR>(s, p, x);
        __syncthreads();
        if (p.has_a) {
            float a[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t at = (p.aj + p.col) * kFlat + p.ai + e / 4 * 8 + p.row + e % 4;
                a[e] = (wide ? s.flat[at] : s.flat[at] + s.flat[at + 32 * kFlat]) * (kScaleX / (kX10 * kX10));
            }
            put_a<PAIR>(s, p, a);
        }
        __syncthreads();
        if (p.has_a) make_b<PAIR>(s, p, m.M, f.b, f.c);
        __syncthreads();
        if (p.has_x) update<PAIR>(s, p, m.M, f.a, x);
    }
    if (step == c.steps) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s.flat[(p.xi + e / 4 * 8 + p.row + e % 4) * kFlat + p.xj + p.col] = x[e];
        __syncthreads();
        put_result<T, MUON>(c, m, s.flat, base, rows, cols, m.scale / kX10);
        return;
    }
    if (p.has_x) {
        put_rows<PAIR>(s, p, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) kept[i * 64 * kWaves] = float4v{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
    }
    __syncthreads();
    if (p.has_a) {
        float a[16];
        gram<PAIR>(s, p, n, a);
        float *const to = grams + ((step & 1u) * strips + t.j) * part + (p.aj + p.col) * side + p.ai + p.row;
#pragma unroll
        for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4v *>(to + e * 2) = float4v{a[e], a[e + 1], a[e + 2], a[e + 3]};
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
template <bool PAIR>
static void thin(const OrthoLayout &lay, const OrthoCall &c, const Polynomial &f, uint32_t step, hipStream_t s)
{
    const dim3 grid(lay.pack.n), block(64 * kWaves);
    if (!c.out) k_ortho_thin<float, true, PAIR><<<grid, block, 0, s>>>(lay, c, f, step);
    else if (lay.type == CO3_F32) k_ortho_thin<float, false, PAIR><<<grid, block, 0, s>>>(lay, c, f, step);
    else if (lay.type == CO3_BF16) k_ortho_thin<__bf16, false, PAIR><<<grid, block, 0, s>>>(lay, c, f, step);
    else k_ortho_thin<_Float16, false, PAIR><<<grid, block, 0, s>>>(lay, c, f, step);
}

hipError_t launch_orthogonalize_small(const OrthoLayout &lay, const OrthoCall &c, hipStream_t s)
{
    ProfScope prof(K_ORTHO_SMALL, s);
    if (lay.products == CO3_PRODUCTS_PAIR) small<true>(lay, c, s);
    else small<false>(lay, c, s);
    return hipGetLastError();
}

hipError_t launch_orthogonalize_thin(const OrthoLayout &lay, const OrthoCall &c, hipStream_t s)
{
    for (uint32_t step = 0; step <= c.steps; ++step) {
        const float *f = c.coefficients + 3 * (step ? step - 1 : 0);
        const Polynomial poly = {f[0], f[1], f[2]};
        ProfScope prof(K_ORTHO_THIN, s);
        if (lay.products == CO3_PRODUCTS_PAIR) thin<true>(lay, c, poly, step, s);
        else thin<false>(lay, c, poly, step, s);
    }
    return hipGetLastError();
}

}  // namespace co3
