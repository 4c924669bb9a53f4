// Products of matrices in 8 bits: out[m][n] = sum over k of A(m, k) B(k, n), both of them e4m3 numbers with a power of two for each block.
//
// A turn takes 128 of k: one block's width, so that every number of a row (of a column, where an operand is read down its rows) has one scale in
// it.  Both operands go to LDS as they lie in memory, in pieces of 128 rows by 128 bytes: 128 rows along the sum, or, of an operand
// whose rows run across the sum, 128 of k by 128 columns, which LDS's transposing read turns as it is read.  So one copy of a matrix serves
// every product that it takes part in.
//
// Numbers.  Results of 16 bits are made by the matrix instructions for 8-bit numbers, which take the scales as they are, powers of two.
// Their sums are not fp32's: sixteen products at a time are aligned to the largest and cut off some 16 bits below it.  Measured
// against 64 bits: 1.4e-5 of the result for normal numbers, 7e-5 for numbers with outliers, where a rounding to bf16 is 1.7e-3.  Results of
// fp32 are made from the same bytes turned into bf16 with their scales, which rounds nothing; the products are exact in fp32, and
// the sums fp32's (1e-7).
#include "blocks8.h"
#include "co3_internal.h"
#include "lds_loads.h"
#include "matmul8.h"
#include "tensor_types.h"

namespace co3 {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int2v __attribute__((ext_vector_type(2)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// The forms of a workgroup: a tile of T x T by WM x WN wavefronts of FM x FN fragments of 32 x 32.
template <int F> struct Form8;
template <> struct Form8<256> { static constexpr int T = 256, WM = 2, WN = 4, FM = 4, FN = 2; };
template <> struct Form8<128> { static constexpr int T = 128, WM = 2, WN = 2, FM = 2, FN = 2; };
template <int F> constexpr int kThreads8 = 64 * Form8<F>::WM * Form8<F>::WN;
constexpr int kPiece = 128 * 128;                                    // bytes of a piece in LDS
template <int F> constexpr int kStage8 = 2 * Form8<F>::T * 128;     // bytes of a turn
constexpr uint32_t kOutside = 0x80000000u;                           // an offset beyond every buffer here

// Where 16 bytes of a piece's row lie in its 128 bytes: exchanged by the row's number, so that the same 16 bytes of eight rows lie in
// different banks, whether eight lanes read them along their rows or sixteen lanes down them.
__device__ inline uint32_t place8(uint32_t row, uint32_t chunk) { return row * 128 + ((chunk ^ (row & 7u)) * 16); }

// What a workgroup reads of an operand.  DOWN: stored [k][its rows].
struct Side {
    const uint8_t *values;     // the tile's first row (column, if DOWN) at k = 0
    const uint8_t *scales;     // at k = 0
    uint32_t ld;
    uint32_t bytes;            // of the buffer from `values` on; if DOWN, of a row's end
    uint32_t wide;             // bytes of a row, rounded up to 16
    uint32_t scale_step;       // from turn to turn
};

template <bool DOWN, int T>
__device__ inline Side side_of(const co3_blocks8 &x, uint32_t i, uint32_t at)
{
    Side s;
    if (x.batch == 1) i = 0;
    s.wide = (x.cols + 15u) & ~15u;
    s.ld = (uint32_t)x.ld;
    s.values = x.values + i * x.batch_stride + (DOWN ? at : at * x.ld);
    s.scales = x.scales + (uint64_t)i * block_columns(x) * x.scale_ld;
    const uint32_t left = (uint32_t)x.rows - at, n = left < (uint32_t)T ? left : (uint32_t)T;
    s.bytes = DOWN ? s.wide - at : (n - 1) * s.ld + s.wide;
    s.scale_step = DOWN ? 1u : x.scale_ld;
    return s;
}

// Where the scale of row `row` (of a column, if DOWN) is at k = 0; that of the last row for those behind it.
template <bool DOWN>
__device__ inline uint32_t scale_at(const co3_blocks8 &x, uint32_t row)
{
    const uint32_t last = DOWN ? x.cols - 1 : (uint32_t)x.rows - 1, r = row < last ? row : last;
    return DOWN ? r / kBlockCols * x.scale_ld : x.block_rows == 1 ? r : r / 128;
}

// 32 bytes of k of a fragment's rows, from k = half 64 + lane / 32 32 on.  `row`: the fragment's first in the tile.
template <bool DOWN>
__device__ inline int8v read_fragment(const unsigned char *tile, int row, int half)
{
    const uint32_t lane = threadIdx.x & 63u;
    int8v v;
    if (DOWN) {   // sixteen lanes read eight rows of k of sixteen columns, and are given eight of one
        typedef __attribute__((address_space(3))) int2v *lds8;
        const uint32_t chunk = (uint32_t)(row % 128) / 16 + lane / 16 % 2;
        const unsigned char *at = tile + row / 128 * kPiece + place8(half * 64 + lane / 32 * 32 + lane % 16 / 2, chunk) + lane % 2 * 8;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int2v r = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds8)(at + j * 8 * 128));
            v[2 * j] = r[0];
            v[2 * j + 1] = r[1];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int4v r = *reinterpret_cast<const int4v *>(tile + row * 128 + place8(lane % 32, half * 4 + lane / 32 * 2 + j));
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * j + e] = r[e];
        }
    }
    return v;
}

// Eight numbers times their scale in bf16.
__device__ inline bf16x8 widen(int low, int high, float scale)
{
    bf16x8 v;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int w = h ? high : low;
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
        v[4 * h] = a[0]; v[4 * h + 1] = a[1]; v[4 * h + 2] = b[0]; v[4 * h + 3] = b[1];
    }
    return v;
}

// Four results next to each other in a row.
template <typename T>
__device__ inline void store_four(T *to, int n, const float *v, bool add)
{
    typename Pack<T, 4>::V p;
    if (add) p = load_pack<T, 4>(to, n);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = (T)(add ? (float)p[i] + v[i] : v[i]);
    store_pack<T, 4>(to, n, p);
}

// A workgroup takes a tile of a matrix of the batch and a slice of its sum.  DM, DN: the operand that has the result's rows, its columns, is
// read down.  EXACT: by way of bf16.  The instructions' rows are the result's columns, so that a lane has four next to each other.
template <typename T, bool DM, bool DN, bool EXACT, int F>
__global__ __launch_bounds__(kThreads8<F>, F == 128 ? 2 : 1) void k_matmul8(co3_matmul8_args a, Matmul8Plan plan, uint32_t first_matrix)
{
    constexpr int S = Form8<F>::T, FM = Form8<F>::FM, FN = Form8<F>::FN, WN = Form8<F>::WN, WAVES = kThreads8<F> / 64;
    constexpr int LOADS = kStage8<F> / 1024 / WAVES, HALF = S * 128;   // of a wavefront in a turn; bytes of an operand
    __shared__ __attribute__((aligned(16))) unsigned char lds[2 * kStage8<F>];
    const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t matrix = first_matrix + blockIdx.y;
    // Workgroups go to the eight XCDs in turn, each with a cache of its own: each takes a neighbourhood, columns of eight tiles' height.
    const uint32_t n = plan.tiles * plan.slices, x = blockIdx.x % 8, q = n / 8 * x + (n % 8 < x ? n % 8 : x) + blockIdx.x / 8;
    const uint32_t slice = q / plan.tiles, tile = q % plan.tiles;
    const uint32_t band = tile / (8 * plan.tiles_n), left_m = plan.tiles_m - band * 8, high = left_m < 8 ? left_m : 8, in = tile - band * 8 * plan.tiles_n;
    const uint32_t m0 = (band * 8 + in % high) * S, n0 = in / high * S;
    const uint32_t begin = plan.turns / plan.slices * slice + (plan.turns % plan.slices < slice ? plan.turns % plan.slices : slice);
    const uint32_t turns = plan.turns / plan.slices + (slice < plan.turns % plan.slices ? 1u : 0u);
    const int wm = (int)(wave / WN) * FM * 32, wn = (int)(wave % WN) * FN * 32;

    const Side sm = side_of<DM, S>(a.a, matrix, m0), sn = side_of<DN, S>(a.b, matrix, n0);
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char *)lds);
    // The wavefront's loads, eight rows of a piece each: the first operand's pieces, then the second's.
    uint32_t offset[LOADS];
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
        const uint32_t load = wave * LOADS + l, of_n = load >= HALF / 1024 ? 1u : 0u, piece = load % (HALF / 1024) / 16, r = load % 16 * 8 + lane / 8;
        const uint32_t chunk = (lane % 8) ^ (r & 7u);
        const Side &s = of_n ? sn : sm;
        if (of_n ? DN : DM) {
            const uint32_t c = piece * 128 + chunk * 16;
            offset[l] = c < s.bytes ? r * s.ld + c : kOutside;
        } else {
            offset[l] = (piece * 128 + r) * s.ld + chunk * 16;   // rows behind the last lie outside
        }
    }
    const auto fetch = [&](uint32_t turn) __attribute__((always_inline)) {
        const uint32_t k = (begin + turn) * 128, to = lds0 + turn % 2 * kStage8<F>;
        const auto side = [&](const Side &s, bool down, uint32_t rows, int from, int till) __attribute__((always_inline)) {
            const uint32_t left = rows - k;   // of k, if down
            const u32x4 base = down ? buffer_of(s.values + (uint64_t)k * s.ld, ((left < 128 ? left : 128) - 1) * s.ld + s.bytes) : buffer_of(s.values, s.bytes);
            const bool ragged = !down && k + 128 > s.wide;
#pragma unroll
            for (int l = 0; l < LOADS; ++l) {
                if (l < from || l >= till) continue;
                uint32_t o = offset[l];
                const uint32_t r = (wave * LOADS + l) % 16 * 8 + lane / 8;
                if (ragged && k + ((lane % 8) ^ (r & 7u)) * 16 >= s.wide) o = kOutside;
                load_to_lds(base, o, down ? 0 : k, to + (wave * LOADS + l) * 1024);
            }
        };
        // a wavefront's loads are all of one operand
        if (wave * LOADS < HALF / 1024) side(sm, DM, (uint32_t)a.a.rows, 0, LOADS);
        else side(sn, DN, (uint32_t)a.b.rows, 0, LOADS);
    };

    uint32_t at_m[FM], at_n[FN];
    uint32_t next_m[FM], next_n[FN], scale_m[FM], scale_n[FN];
#pragma unroll
    for (int i = 0; i < FM; ++i) at_m[i] = scale_at<DM>(a.a, m0 + wm + i * 32 + lane % 32);
#pragma unroll
    for (int j = 0; j < FN; ++j) at_n[j] = scale_at<DN>(a.b, n0 + wn + j * 32 + lane % 32);
    const auto fetch_scales = [&](uint32_t turn) __attribute__((always_inline)) {
        const uint8_t *pm = sm.scales + (uint64_t)(begin + turn) * sm.scale_step, *pn = sn.scales + (uint64_t)(begin + turn) * sn.scale_step;
#pragma unroll
        for (int i = 0; i < FM; ++i) next_m[i] = pm[at_m[i]];
#pragma unroll
        for (int j = 0; j < FN; ++j) next_n[j] = pn[at_n[j]];
    };

    float16v acc[FM][FN] = {};
    fetch_scales(0);
    fetch(0);
    for (uint32_t t = 0; t < turns; ++t) {
        wait_loads<0>();
        meet();   // this turn is there, and all have read the one before it
#pragma unroll
        for (int i = 0; i < FM; ++i) { scale_m[i] = next_m[i]; asm volatile("" : "+v"(scale_m[i])); }
#pragma unroll
        for (int j = 0; j < FN; ++j) { scale_n[j] = next_n[j]; asm volatile("" : "+v"(scale_n[j])); }
        if (t + 1 < turns) {
            fetch_scales(t + 1);
            fetch(t + 1);
        }
        const unsigned char *pm = lds + t % 2 * kStage8<F>, *pn = pm + HALF;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int8v vm[FM], vn[FN];
#pragma unroll
            for (int j = 0; j < FN; ++j) vn[j] = read_fragment<DN>(pn, wn + j * 32, h);
#pragma unroll
            for (int i = 0; i < FM; ++i) vm[i] = read_fragment<DM>(pm, wm + i * 32, h);
            if constexpr (!EXACT) {
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(vn[j], vm[i], acc[i][j], 0, 0, 0, (int)scale_n[j], 0, (int)scale_m[i]);
            } else {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    bf16x8 wn_[FN], wm_[FM];
#pragma unroll
                    for (int j = 0; j < FN; ++j) wn_[j] = widen(vn[j][2 * g], vn[j][2 * g + 1], power_of(scale_n[j]));
#pragma unroll
                    for (int i = 0; i < FM; ++i) wm_[i] = widen(vm[i][2 * g], vm[i][2 * g + 1], power_of(scale_m[i]));
#pragma unroll
                    for (int i = 0; i < FM; ++i)
#pragma unroll
                        for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wn_[j], wm_[i], acc[i][j], 0, 0, 0);
                }
            }
        }
    }

    const bool whole = plan.slices == 1;
    float *part = static_cast<float *>(a.workspace) + ((uint64_t)slice * plan.batch + matrix) * plan.m * plan.part_ld;
    T *out = static_cast<T *>(a.out) + matrix * a.out_batch_stride;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const uint32_t m = m0 + wm + i * 32 + lane % 32;
        if (m >= plan.m) continue;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t c = n0 + wn + j * 32 + e * 8 + lane / 32 * 4;
                if (c >= plan.n) continue;
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = acc[i][j][4 * e + k];
                if (whole) store_four<T>(out + m * a.out_stride + c, (int)(plan.n - c), v, a.accumulate);
                else *reinterpret_cast<float4 *>(part + (uint64_t)m * plan.part_ld + c) = make_float4(v[0], v[1], v[2], v[3]);
            }
    }
}

// The slices of a sum, in their order; zeros for none.
template <typename T>
__global__ __launch_bounds__(256) void k_matmul8_join(co3_matmul8_args a, Matmul8Plan plan, uint64_t first)
{
    const uint64_t fours = plan.part_ld / 4, i = first + (uint64_t)blockIdx.x * 256 + threadIdx.x, each = fours * plan.m;
    if (i >= each * plan.batch) return;
    const uint32_t matrix = (uint32_t)(i / each), m = (uint32_t)(i % each / fours), c = (uint32_t)(i % fours) * 4;
    const float *part = static_cast<const float *>(a.workspace) + ((uint64_t)matrix * plan.m + m) * plan.part_ld + c;
    float v[4] = {};
    for (uint32_t s = 0; s < plan.slices; ++s) {
        const float4 p = *reinterpret_cast<const float4 *>(part + (uint64_t)s * plan.batch * plan.m * plan.part_ld);
        v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
    }
    store_four<T>(static_cast<T *>(a.out) + matrix * a.out_batch_stride + m * a.out_stride + c, (int)(plan.n - c), v, a.accumulate);
}

template <typename T, bool DM, bool DN, int F>
static void multiply(const co3_matmul8_args &a, const Matmul8Plan &plan, hipStream_t s)
{
    const uint32_t groups = plan.tiles * plan.slices;
    const uint64_t room = ((1ull << 32) - 1) / kThreads8<F> / groups, most = room < 65535 ? room : 65535;   // matrices of a launch: at least one (plan_matmul8)
    for (uint32_t i = 0; i < plan.batch; i += (uint32_t)most) {
        const uint32_t count = (uint32_t)(plan.batch - i < most ? plan.batch - i : most);
        k_matmul8<T, DM, DN, sizeof(T) == 4, F><<<dim3(groups, count), dim3(kThreads8<F>), 0, s>>>(a, plan, i);
    }
}

template <typename T, int F>
static void multiply_of(const co3_matmul8_args &a, const Matmul8Plan &plan, hipStream_t s)
{
    if (a.transpose_a) a.transpose_b ? multiply<T, true, false, F>(a, plan, s) : multiply<T, true, true, F>(a, plan, s);
    else a.transpose_b ? multiply<T, false, false, F>(a, plan, s) : multiply<T, false, true, F>(a, plan, s);
}

template <typename T>
static void matmul8_of(const co3_matmul8_args &a, const Matmul8Plan &plan, hipStream_t s)
{
    if (plan.slices) {
        ProfScope prof(K_MATMUL8, s);
        if (plan.form == 256) multiply_of<T, 256>(a, plan, s);
        else multiply_of<T, 128>(a, plan, s);
    }
    if (plan.slices == 1 || (plan.slices == 0 && a.accumulate)) return;
    ProfScope prof(K_MATMUL8_JOIN, s);
    const uint64_t all = (uint64_t)plan.batch * plan.m * (plan.part_ld / 4), most = (((1ull << 32) - 1) / 256) * 256;
    for (uint64_t i = 0; i < all; i += most) {
        const uint64_t n = all - i < most ? all - i : most;
        k_matmul8_join<T><<<dim3((uint32_t)((n + 255) / 256)), dim3(256), 0, s>>>(a, plan, i);
    }
}

hipError_t launch_matmul8(const co3_matmul8_args &a, const Matmul8Plan &plan, hipStream_t s)
{
    if (a.type == CO3_F32) matmul8_of<float>(a, plan, s);
    else if (a.type == CO3_BF16) matmul8_of<__bf16>(a, plan, s);
    else matmul8_of<_Float16>(a, plan, s);
    return hipGetLastError();
}

}  // namespace co3
