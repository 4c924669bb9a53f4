// Products of matrices in 8 bits: out[m][n] = sum over k of A(m, k) B(k, n), both of them e4m3 numbers with a power of two for each block.
//
// A turn takes 128 of k: one block's width, so that every number of a row (of a column, where an operand is read down its rows) has one scale in
// it.  Both operands go to LDS as they lie in memory, in pieces of 128 rows by 128 bytes: 128 rows along the sum, or, of an operand
// whose rows run across the sum, 128 of k by 128 columns, which LDS's transposing read turns as it is read.  So one copy of a matrix serves
// every product that it takes part in.
//
// Numbers.  Results of 16 bits are made by the matrix instructions for 8-bit numbers, which take the scales as they are, powers of two.
// Their sums are not fp32's: sixteen products at a time are aligned to the largest and cut off some 16 bits below it.  Measured
// against 64 bits: 1.3e-5 to 1.5e-5 of the result for normal numbers, 4e-5 to 8e-5 for numbers with outliers, where a rounding to bf16 is 1.7e-3.  Results of
// fp32 are made from the same bytes turned into bf16 with their scales, which rounds nothing; the products are exact in fp32, and
// the sums fp32's (1e-7), at half of the rate.
//
// Measured (MI355X, normal numbers; the library's product of 8192 x 8192 e4m3 numbers with one scale 2.81 PFLOP/s, of bf16 1.54): 8192 x 4096 x 4096
// to bf16 118 us a call = 2.33 PFLOP/s, 122 to 127 in the profiler; there 8192^3 453 to 467 us = 2.43 to 2.35, gradients of 4 x 4096^3 to bf16 246 to 255 us = 2.2 and
// to fp32 442 to 461 us = 1.2 PFLOP/s.  The matrix instructions are busy for 52, 56 and 63 % of the cycles (the first, the gradients), at 2 GHz; a
// wavefront waits for loads, LDS and the others for a third of its time.  Four wavefronts of 128 x 128 a tile took 143 us where eight took 127, and
// scales read earlier spill (317 us for 255 with b read down).  One row by 4096 x 4096 is bound by the reading of b and a launch: 6.2 us a call, 2.7 TB/s.
#include "blocks8.h"
#include "co3_internal.h"
#include "lds_loads.h"
#include "matmul8.h"
#include "tensor_types.h"

namespace co3 {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// The forms of a workgroup: a tile of T x T by WM x WN wavefronts of FM x FN fragments of 32 x 32, RING turns of it in LDS.
template <int F> struct Form8;
template <> struct Form8<256> { static constexpr int T = 256, WM = 2, WN = 4, FM = 4, FN = 2, RING = 2, GROUPS = 1; };
template <> struct Form8<128> { static constexpr int T = 128, WM = 2, WN = 2, FM = 2, FN = 2, RING = 2, GROUPS = 2; };
template <> struct Form8<64> { static constexpr int T = 64, WM = 2, WN = 2, FM = 1, FN = 1, RING = 4, GROUPS = 2; };
template <int F> constexpr int kThreads8 = 64 * Form8<F>::WM * Form8<F>::WN;
template <int F> constexpr int kOperand8 = Form8<F>::T * 128;                               // bytes of an operand's numbers in a turn
template <int F> constexpr int kStage8 = 2 * kOperand8<F> + 2 * Form8<F>::T * 4;            // bytes of a turn: a word with its scale for each row
constexpr uint32_t kOutside = 0x80000000u;                                                  // an offset beyond every buffer here

// A turn's numbers of an operand lie in LDS in pieces of 128 rows by 128 bytes: rows along the sum, or (DOWN) 128 of k by 128 of the rows; at 64
// rows, of 64 by 128 or 128 by 64.  Where 16 bytes of a piece's row lie is exchanged by the row's number, so that what is read at a time lies in
// different ones of the 64 banks: the same 16 bytes of sixteen rows along the sum; down them, 32 bytes of eight rows.
template <bool DOWN, int WIDTH>
__device__ inline uint32_t exchanged(uint32_t row, uint32_t chunk) { return !DOWN ? chunk ^ (row >> 1 & 7u) : WIDTH == 128 ? chunk ^ (row & 7u) : chunk ^ (row >> 1 & 3u); }

__device__ inline uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }

// Where the scale of a row (DOWN: of a column) is at k = 0; that of the last one for those behind it.
template <bool DOWN>
__device__ inline uint32_t scale_at(const co3_blocks8 &x, uint32_t row)
{
    const uint32_t last = DOWN ? x.cols - 1 : (uint32_t)x.rows - 1, r = row < last ? row : last;
    return DOWN ? r / kBlockCols * x.scale_ld : x.block_rows == 1 ? r : r / 128;
}

// What a wavefront asks for of its operand in a turn: LOADS times a kilobyte, and a word of scales a lane.  Without a branch, whatever the operand
// (down: stored [k][its rows]), the turn and the wavefront: with one in a turn the compiler put all of its products at the end, and had too few registers.
struct Side {
    const uint8_t *values, *scales;   // the tile's first row (column, if down) at k = 0; the matrix's scales
    uint32_t bytes, limit, rows;      // bytes: of the buffer from `values` on, if down of a row's end; where a row ends, if not down; of k, if down
    uint32_t down, along;             // from k to k if down, and along a row if not: the other is 0
    uint32_t offset, odd, place;      // this lane's of the wavefront's even loads; how much further odd ones'; its place of 16 bytes along a row
    uint32_t next;                    // from load to load
    uint32_t at, all, step, words;    // this lane's word of scales; bytes of all; from turn to turn; which turns have words of their own

    // `load`: the wavefront's first of the operand's; `row`: the lane's, whose scale it asks for
    template <bool DOWN, int T>
    __device__ inline void init(const co3_blocks8 &x, uint32_t i, uint32_t first, uint32_t load, uint32_t row)
    {
        constexpr int WIDTH = DOWN && T == 64 ? 64 : 128, ROWS = 1024 / WIDTH, PIECE = T == 64 ? 8 : 16;   // of a load; loads of a piece
        const uint32_t lane = threadIdx.x & 63u, wide = (x.cols + 15u) & ~15u, left = (uint32_t)x.rows - first, n = left < (uint32_t)T ? left : (uint32_t)T;
        if (x.batch == 1) i = 0;
        const uint32_t ld = (uint32_t)x.ld;
        down = DOWN ? ld : 0;
        along = DOWN ? 0 : 128;
        values = x.values + i * x.batch_stride + (DOWN ? first : first * x.ld);
        bytes = DOWN ? wide - first : (n - 1) * ld + wide;
        limit = DOWN ? 0xffffffffu : wide;
        rows = (uint32_t)x.rows;
        next = ROWS * ld;
        const uint32_t r = lane / (WIDTH / 16), chunk = exchanged<DOWN, WIDTH>(r, lane % (WIDTH / 16)), column = load / PIECE * 128 + chunk * 16;
        if (DOWN) offset = column < bytes ? (load % PIECE * ROWS + r) * ld + column : kOutside;
        else offset = (load * ROWS + r) * ld + chunk * 16;   // rows behind the last lie outside
        place = DOWN ? 0 : chunk * 16;
        odd = DOWN ? 0 : chunk < 4 ? 64 : 0u - 64;           // the exchange of a row 8 further: `load` is even
        const uint32_t columns = block_columns(x);
        all = columns * x.scale_ld;
        scales = x.scales + (uint64_t)i * all;
        at = scale_at<DOWN>(x, first + row) & ~3u;
        step = DOWN ? 1 : x.scale_ld;
        words = DOWN ? ~3u : ~0u;
    }
    // Part `part` of PARTS of a turn's loads; the last one asks for the scales too.  Turns from `end` on: zeros, from nowhere.
    template <int LOADS, int PARTS>
    __device__ inline void fetch(uint32_t turn, uint32_t end, uint32_t to, uint32_t to_scales, int part) const
    {
        const uint32_t k = turn * 128, left = rows - k, high = left < 128 ? left : 128, none = turn < end ? ~0u : 0u;
        const u32x4 from = buffer_of(values + (uint64_t)k * down, ((high - 1) * down + bytes) & none);
        const uint32_t o[2] = {k + place >= limit ? kOutside : offset, k + place + odd >= limit ? kOutside : offset + odd};
#pragma unroll
        for (int l = 0; l < LOADS; ++l)
            if (l * PARTS / LOADS == part) load_to_lds(from, o[l % 2], uniform(turn * along + l * next), to + l * 1024);
        if (part == PARTS - 1) load_word_to_lds(buffer_of(scales, all & none), at, uniform((turn & words) * step), to_scales);
    }
};

// 32 bytes of k of a fragment's rows, from k = half 64 + lane / 32 32 on.  `row`: the fragment's first in the tile.
template <bool DOWN, int T>
__device__ inline int8v read_fragment(const unsigned char *tile, int row, int half)
{
    const uint32_t lane = threadIdx.x & 63u;
    int8v v;
    if (DOWN) {   // sixteen lanes read eight rows of k of sixteen columns, and are given eight of one
        constexpr int WIDTH = T == 64 ? 64 : 128;
        typedef __attribute__((address_space(3))) int2v *lds8;
        const uint32_t chunk = (uint32_t)(row % WIDTH) / 16 + lane / 16 % 2, k = half * 64 + lane / 32 * 32 + lane % 16 / 2;
        const unsigned char *at = tile + row / 128 * 128 * 128 + k * WIDTH + exchanged<DOWN, WIDTH>(k, chunk) * 16 + lane % 2 * 8;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int2v r = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds8)(at + j * 8 * WIDTH));
            v[2 * j] = r[0];
            v[2 * j + 1] = r[1];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int4v r = *reinterpret_cast<const int4v *>(tile + (row + lane % 32) * 128 + exchanged<DOWN, 128>(lane, half * 4 + lane / 32 * 2 + j) * 16);
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

// Results next to each other in a row.
template <typename T, int N>
__device__ inline void store_results(T *to, int n, const float *v, bool add)
{
    typename Pack<T, N>::V p;
    if (add) p = load_pack<T, N>(to, n);
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = (T)(add ? (float)p[i] + v[i] : v[i]);
    store_pack<T, N>(to, n, p);
}

// A workgroup takes a tile of a matrix of the batch and a slice of its sum.  DM, DN: the operand that has the result's rows, its columns, is
// read down.  EXACT: by way of bf16.  The instructions' rows are the result's columns, so that a lane has four next to each other.
// While half a turn is multiplied, the next half is read from LDS; the turns behind it are on their way to LDS.
template <typename T, bool DM, bool DN, bool EXACT, int F>
__global__ __launch_bounds__(kThreads8<F>, Form8<F>::GROUPS * kThreads8<F> / 256) void k_matmul8(co3_matmul8_args a, Matmul8Plan plan, uint32_t first_matrix)
{
    constexpr int S = Form8<F>::T, FM = Form8<F>::FM, FN = Form8<F>::FN, WN = Form8<F>::WN, RING = Form8<F>::RING, WAVES = kThreads8<F> / 64;
    constexpr int LOADS = 2 * kOperand8<F> / 1024 / WAVES, ASKED = LOADS + 1;   // of a wavefront in a turn
    constexpr int PITCH = FN * 32 + 4;   // floats of a row of results in LDS: sixteen bytes of eight rows lie in different banks
    constexpr size_t kTurns = (size_t)RING * kStage8<F>, kResults = (size_t)WAVES * 32 * PITCH * sizeof(float);
    __shared__ __attribute__((aligned(16))) unsigned char lds[kTurns > kResults ? kTurns : kResults];
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

    // A wavefront's loads are all of one operand: the first half's of the first.
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) unsigned char *)lds);
    const bool of_n = wave >= WAVES / 2;
    const uint32_t load = wave % (WAVES / 2) * LOADS, word = wave % (WAVES / 2) * 64 % S;   // words: 64 rows a wavefront, the same ones twice where there are fewer
    Side side;
    if (of_n) side.init<DN, S>(a.b, matrix, n0, load, word + lane);
    else side.init<DM, S>(a.a, matrix, m0, load, word + lane);
    const uint32_t to = lds0 + (of_n ? kOperand8<F> : 0) + load * 1024, words = lds0 + 2 * kOperand8<F> + (of_n ? S * 4 : 0) + word * 4;
    const auto fetch = [&](uint32_t turn, int part) __attribute__((always_inline)) {
        const uint32_t stage = turn % RING * kStage8<F>;
        side.fetch<LOADS, FM>(begin + turn, begin + turns, uniform(to + stage), uniform(words + stage), part);
    };
    // Which byte of its word a row's scale is.
    uint32_t shift_m[FM], shift_n[FN];
#pragma unroll
    for (int i = 0; i < FM; ++i) shift_m[i] = DM ? 0 : scale_at<DM>(a.a, m0 + wm + i * 32 + lane % 32) % 4 * 8;
#pragma unroll
    for (int j = 0; j < FN; ++j) shift_n[j] = DN ? 0 : scale_at<DN>(a.b, n0 + wn + j * 32 + lane % 32) % 4 * 8;

    float16v acc[FM][FN] = {};
    int8v vm[FM], vn[FN];
    uint32_t scale_m[FM], scale_n[FN];
    const auto read_m = [&](uint32_t turn, int h, int i) __attribute__((always_inline)) {
        return read_fragment<DM, S>(lds + turn % RING * kStage8<F>, wm + i * 32, h);
    };
    const auto read_n = [&](uint32_t turn, int h, int j) __attribute__((always_inline)) {
        return read_fragment<DN, S>(lds + turn % RING * kStage8<F> + kOperand8<F>, wn + j * 32, h);
    };
    const auto words_of = [&](uint32_t turn) { return reinterpret_cast<const uint32_t *>(lds + turn % RING * kStage8<F> + 2 * kOperand8<F>); };
    const auto read_scales = [&](uint32_t turn) __attribute__((always_inline)) {
        const uint32_t down = (begin + turn) % 4 * 8;
#pragma unroll
        for (int i = 0; i < FM; ++i) scale_m[i] = words_of(turn)[wm + i * 32 + lane % 32] >> (DM ? down : shift_m[i]);
#pragma unroll
        for (int j = 0; j < FN; ++j) scale_n[j] = words_of(turn)[S + wn + j * 32 + lane % 32] >> (DN ? down : shift_n[j]);
    };
    // Half a turn's products; half `h` of `turn` is read meanwhile, a fragment into the registers of the one that was used last (behind the
    // last turn what is left in LDS, unused).  `ask`: a turn's loads too.
    const auto multiply = [&](uint32_t turn, int h, uint32_t ask) __attribute__((always_inline)) {
        int8v next[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) next[j] = read_n(turn, h, j);
        bf16x8 pn[EXACT ? FN : 1][4];
        if constexpr (EXACT) {
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) pn[j][g] = widen(vn[j][2 * g], vn[j][2 * g + 1], power_of(scale_n[j] & 255u));
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            if constexpr (!EXACT) {
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(vn[j], vm[i], acc[i][j], 0, 0, 0, (int)scale_n[j], 0, (int)scale_m[i]);
            } else {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const bf16x8 pm = widen(vm[i][2 * g], vm[i][2 * g + 1], power_of(scale_m[i] & 255u));
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pn[j][g], pm, acc[i][j], 0, 0, 0);
                }
            }
            vm[i] = read_m(turn, h, i);
            __builtin_amdgcn_sched_barrier(0);
            if (h == 0) fetch(ask, i);
        }
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int j = 0; j < FN; ++j) vn[j] = next[j];
    };

#pragma unroll
    for (uint32_t t = 0; t < RING; ++t)
#pragma unroll
        for (int i = 0; i < FM; ++i) fetch(t, i);
    wait_loads<(RING - 1) * ASKED>();
    meet();
    read_scales(0);
#pragma unroll
    for (int j = 0; j < FN; ++j) vn[j] = read_n(0, 0, j);
#pragma unroll
    for (int i = 0; i < FM; ++i) vm[i] = read_m(0, 0, i);
    for (uint32_t t = 0; t < turns; ++t) {
        multiply(t, 1, 0);
        wait_loads<(RING - 2) * ASKED>();
        meet();   // the next turn is there, and all have read this one
        multiply(t + 1, 0, t + RING);
        read_scales(t + 1);
    }
    wait_loads<0>();
    meet();

    // Results go through the wavefront's own place in LDS, 32 rows at a time, so that a row's are stored side by side.
    const bool whole = plan.slices == 1;
    float *part = static_cast<float *>(a.workspace) + ((uint64_t)slice * plan.batch + matrix) * plan.m * plan.part_ld;
    T *out = static_cast<T *>(a.out) + matrix * a.out_batch_stride;
    float *own = reinterpret_cast<float *>(lds) + wave * 32 * PITCH;
    constexpr int LANES = FN * 32 / 8;   // of a row, eight results each
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<float4 *>(own + lane % 32 * PITCH + j * 32 + e * 8 + lane / 32 * 4) =
                    make_float4(acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]);
#pragma unroll
        for (int r = 0; r < 32; r += 64 / LANES) {
            const uint32_t row = r + lane / LANES, m = m0 + wm + i * 32 + row, c = n0 + wn + lane % LANES * 8;
            const float *from = own + row * PITCH + lane % LANES * 8;
            const float4 low = *reinterpret_cast<const float4 *>(from), high = *reinterpret_cast<const float4 *>(from + 4);
            if (m >= plan.m || c >= plan.n) continue;
            const float v[8] = {low.x, low.y, low.z, low.w, high.x, high.y, high.z, high.w};
            if (whole) store_results<T, 8>(out + m * a.out_stride + c, (int)(plan.n - c), v, a.accumulate);
            else store_results<float, 8>(part + (uint64_t)m * plan.part_ld + c, (int)(plan.n - c), v, false);
        }
    }
}

// Products of few rows, both operands along their rows: reading b is all there is.  A workgroup takes sixteen of b's rows, its wavefronts
// every eighth turn each, four turns on their way at a time from memory to the registers that the instructions read; the wavefronts' sums meet
// in LDS.
template <typename T, bool EXACT>
__global__ __launch_bounds__(512) void k_matmul8_rows(co3_matmul8_args a, Matmul8Plan plan, uint32_t first_matrix)
{
    constexpr int AHEAD = 4;
    __shared__ float red[8][16][17];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, matrix = first_matrix + blockIdx.y, n0 = blockIdx.x * 16, row = lane % 16, k0 = lane / 16 * 32;
    const uint32_t ma = a.a.batch > 1 ? matrix : 0, mb = a.b.batch > 1 ? matrix : 0, wide = (a.a.cols + 15u) & ~15u;
    const uint8_t *scales_m = a.a.scales + (uint64_t)ma * block_columns(a.a) * a.a.scale_ld + scale_at<false>(a.a, row);
    const uint8_t *scales_n = a.b.scales + (uint64_t)mb * block_columns(a.b) * a.b.scale_ld + scale_at<false>(a.b, n0 + row);
    const bool in_m = row < plan.m, in_n = n0 + row < plan.n;
    const uint8_t *pm = a.a.values + ma * a.a.batch_stride + (in_m ? row : 0) * a.a.ld + k0, *pn = a.b.values + mb * a.b.batch_stride + (uint64_t)(in_n ? n0 + row : 0) * a.b.ld + k0;
    float4v acc = {};
    for (uint32_t t = wave; t < plan.turns; t += 8 * AHEAD) {
        int4v vm[AHEAD][2], vn[AHEAD][2];
        uint32_t scale_m[AHEAD], scale_n[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const uint32_t turn = t + 8 * i, k = turn * 128;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool in = turn < plan.turns && k + k0 + h * 16 < wide;
                vn[i][h] = vm[i][h] = int4v{};
                if (in && in_n) vn[i][h] = *reinterpret_cast<const int4v *>(pn + k + h * 16);
                if (in && in_m) vm[i][h] = *reinterpret_cast<const int4v *>(pm + k + h * 16);
            }
            scale_n[i] = scale_m[i] = 127;
            if (turn < plan.turns) {
                scale_n[i] = scales_n[(uint64_t)turn * a.b.scale_ld];
                scale_m[i] = scales_m[(uint64_t)turn * a.a.scale_ld];
            }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {   // turns behind the last add zeros
            const int8v bm = __builtin_shufflevector(vm[i][0], vm[i][1], 0, 1, 2, 3, 4, 5, 6, 7), bn = __builtin_shufflevector(vn[i][0], vn[i][1], 0, 1, 2, 3, 4, 5, 6, 7);
            if constexpr (!EXACT) {
                acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(bn, bm, acc, 0, 0, 0, (int)scale_n[i], 0, (int)scale_m[i]);
            } else {
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(bn[2 * g], bn[2 * g + 1], power_of(scale_n[i])), widen(bm[2 * g], bm[2 * g + 1], power_of(scale_m[i])),
                                                                  acc, 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) red[wave][lane % 16][lane / 16 * 4 + e] = acc[e];
    __syncthreads();
    const uint32_t m = threadIdx.x / 16, c = threadIdx.x % 16;
    if (m >= plan.m || n0 + c >= plan.n) return;   // m < 32
    float v = red[0][m][c];
#pragma unroll
    for (int w = 1; w < 8; ++w) v += red[w][m][c];
    store_results<T, 1>(static_cast<T *>(a.out) + matrix * a.out_batch_stride + m * a.out_stride + n0 + c, 1, &v, a.accumulate);
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
    store_results<T, 4>(static_cast<T *>(a.out) + matrix * a.out_batch_stride + m * a.out_stride + c, (int)(plan.n - c), v, a.accumulate);
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
static void multiply_rows(const co3_matmul8_args &a, const Matmul8Plan &plan, hipStream_t s)
{
    const uint64_t room = ((1ull << 32) - 1) / 512 / plan.tiles, most = room < 65535 ? room : 65535;
    for (uint32_t i = 0; i < plan.batch; i += (uint32_t)most) {
        const uint32_t count = (uint32_t)(plan.batch - i < most ? plan.batch - i : most);
        k_matmul8_rows<T, sizeof(T) == 4><<<dim3(plan.tiles, count), dim3(512), 0, s>>>(a, plan, i);
    }
}

template <typename T>
static void matmul8_of(const co3_matmul8_args &a, const Matmul8Plan &plan, hipStream_t s)
{
    if (plan.slices) {
        ProfScope prof(K_MATMUL8, s);
        if (plan.form == kFormRows) multiply_rows<T>(a, plan, s);
        else if (plan.form == 256) multiply_of<T, 256>(a, plan, s);
        else if (plan.form == 128) multiply_of<T, 128>(a, plan, s);
        else multiply_of<T, 64>(a, plan, s);
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
