// Newton-Schulz iteration of every matrix of a flat vector, and the update that Muon makes of it.
//
//   X_0 = G / (|G|_F + eps);   A = X X^T,  B = b A + c A A,  X <- a X + B X
//
// A launch does one product for all matrices, a workgroup one tile: tables made with the plan say which.  A and A A are
// symmetric: only tiles on and below the diagonal are computed, the others are written from them.  Their operands' rows run along
// the sum; in B X those of X run across it, and are transposed as they are read from LDS.
//
// Numbers.  The matrix instructions take fp16 and add in fp32.  X, A and B are held times 2^14, 2^14 and 2^13: X's singular
// values stay below 2 and B's below 7, so nothing overflows, and at 2^14 what matters is far from the smallest fp16 number
// (of 4096 x 25088 noise, X_0's entries are 1.6 on average).  Scales are powers of two: they round nothing.  X is a pair
// hi + lo of 22 bits, since small singular values grow up to a^steps times (485 at five steps of Muon's a = 3.4445)
// while large ones stay: the rounding of the iterate to 11 bits, spread over all directions, grows with them (a
// matrix of one dominant direction and 10^-3 noise: 9e-2 off, with the pair 2e-4).  The operands of the products are pairs too, unless the
// caller asks for their high parts alone: where the singular values are small, so are A and B beside a, and their roundings do not
// grow (2e-3 off, the size of bf16's own rounding; a few elements, whose roundings do not average out, up to 1.5e-2).
//
// Measured (MI355X; a large copy runs at 4.8 TB/s, the library's fp16 product of 4096 x 4096 at 1.37 PFLOP/s in 100 us):
// one product B X of 4096 x 4096 in pairs 345 us = 1.19 PFLOP/s, of 4096 x 25088 1.14; from high parts alone 140 us = 0.98 PFLOP/s, of which
// 120 us are the sums.  The chip lowers its clock to 1.5 GHz under it: with no loads and no reads of LDS at all the same matrix
// instructions take 94 us.  A product of a few hundred tiles (10 to 30 us) is bound by what a CU gets from the caches, whatever the tile, and by
// what comes before its first turn and behind its last: first loads, the old X, the split, the stores.  Norm and layout are bound by memory.
#include <type_traits>

#include "co3_internal.h"
#include "ortho_device.h"

namespace co3 {

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
// those of g + beta m, are what is summed.  One pass: 25 million elements with momentum 55 us = 5.5 TB/s.
template <typename T, bool MUON>
__global__ __launch_bounds__(256) void k_ortho_norm(OrthoLayout lay, OrthoCall c)
{
    __shared__ double lds[4];
    const PartDev part = lay.parts[blockIdx.x];
    const MatDev m = lay.mats[part.mat];
    constexpr int V = kVec<T>;
    double s = 0.0;
    // 2^share threads a line, as many as it has packs: a part of short lines, a matrix's among others in the same rows, has many of them.  65536
    // lines of one element, two apart: 31 us, 3535 us by one line after the other; of 64 elements, 128 apart, 11 and 90 us.
    uint32_t share = 8;
    while (share && part.len <= (uint64_t)V << (share - 1)) --share;
    for (uint32_t l = threadIdx.x >> share; l < part.lines; l += 256u >> share) {
        const uint64_t at = m.offset + part.at + l * m.ld;
        for (uint64_t k = (uint64_t)(threadIdx.x & ((1u << share) - 1)) * V; k < part.len; k += (uint64_t)V << share) {
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

// Where eight values from column k (a multiple of 8) of row r of a plane of K columns begin.  A plane is made of blocks of 16 rows by
// 64 bytes, a kilobyte each, which is what a wavefront asks for with one load: 32 values, or 16 high and 16 low parts.
template <bool PAIR>
__device__ inline uint64_t place(uint32_t r, uint32_t k, uint32_t K)
{
    constexpr uint32_t D = PAIR ? 16 : 32;
    return ((uint64_t)(r / 16) * (K / D) + k / D) * 512 + r % 16 * 32 + k % D;
}

// What a tile of 64 x 64 floats in LDS is read and written by: 65 words a row, so that neither eight columns of eight rows nor
// eight rows of eight columns meet in a bank.
constexpr int kPitch = 65;

// X_0, with the padding; through LDS, since a tall matrix is laid out by its columns.  25 million elements of an update 67 us = 4.5 TB/s.
template <typename T, bool MUON, bool PAIR>
__global__ __launch_bounds__(256) void k_ortho_pack(OrthoLayout lay, OrthoCall c)
{
    __shared__ double lds[4];
    __shared__ float tile[kBlock * kPitch];
    const TileDev t = lay.pack.tiles[blockIdx.x];
    const MatDev m = lay.mats[t.mat];
    double s = 0.0;
    for (uint32_t p = threadIdx.x; p < m.nparts; p += 256) s += c.partial[m.part + p];
    s = block_sum(s, lds);
    const double f = scale_of(s, c.eps);
    if (f != f && t.i == 0 && t.j == 0 && threadIdx.x == 0) count_not_finite(c);

    for (uint32_t k = blockIdx.x * 256 + threadIdx.x; k < lay.slices; k += gridDim.x * 256) c.counters[k] = 0u;

    const uint32_t gr = (m.tall ? t.j : t.i) * kBlock, gc = (m.tall ? t.i : t.j) * kBlock;   // in the caller's matrix
    const uint32_t lane = threadIdx.x & 63u;
    for (uint32_t r = threadIdx.x >> 6; r < kBlock; r += 4) {
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
    _Float16 *x = c.planes + m.x;
#pragma unroll
    for (uint32_t pass = 0; pass < 2; ++pass) {   // X's rows: the tile's, or its columns
        const uint32_t r = pass * 32 + threadIdx.x / 8, k = threadIdx.x % 8 * 8;
        half8 hi, lo;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            _Float16 h, l;
            split(tile[m.tall ? (k + i) * kPitch + r : r * kPitch + k + i], h, l);
            hi[i] = h;
            lo[i] = l;
        }
        _Float16 *to = x + place<PAIR>(t.i * kBlock + r, t.j * kBlock + k, m.Np);
        *reinterpret_cast<half8 *>(to) = hi;
        *reinterpret_cast<half8 *>(to + (PAIR ? 16 : (uint64_t)m.Mp * m.Np)) = lo;
    }
}

// ---- products -----------------------------------------------------------------------------------------------

enum { GRAM, SQUARE, PRODUCT, LAST };

// The forms of a workgroup: a tile of T x T by WI x WJ wavefronts of FI x FJ fragments of 32 x 32, KW times over: each of these groups
// takes every KW-th turn of the sum.  One group where there are tiles for all CUs; more of them keep more loads on their way.
template <int F> struct Form;
template <> struct Form<256> { static constexpr int T = 256, WI = 2, WJ = 4, FI = 4, FJ = 2, KW = 1; };
template <> struct Form<128> { static constexpr int T = 128, WI = 2, WJ = 2, FI = 2, FJ = 2, KW = 1; };
template <> struct Form<kForm128Twice> { static constexpr int T = 128, WI = 2, WJ = 2, FI = 2, FJ = 2, KW = 2; };
template <> struct Form<64> { static constexpr int T = 64, WI = 2, WJ = 2, FI = 1, FJ = 1, KW = 4; };
template <int F> constexpr int kThreads = 64 * Form<F>::WI * Form<F>::WJ * Form<F>::KW;
// A turn takes 64 bytes of every row of P and of Q: 32 values, or 16 pairs.  LDS holds four turns.
template <bool PAIR> constexpr int kDepth = PAIR ? 16 : 32;
constexpr int kTurn = 32, kRing = 4;                  // fp16 numbers of a row in a turn; turns in LDS
template <int F> constexpr int kStage = 2 * Form<F>::T * kTurn;   // fp16 numbers of a turn

// Where 16 bytes of a row lie in its 64 bytes in LDS: exchanged by the row's number, so that the same 16 bytes of sixteen rows, which
// sixteen lanes read at a time, lie in different ones of the 64 banks.
__device__ inline int exchanged(int row, int chunk) { return chunk ^ (row >> 2 & 3); }

// 64 lanes' 16 bytes from memory to LDS, without a register in between: from base + offset (of every lane) + k, to `lds` + 16 lane.
// Written out, since the compiler would wait for all loads to LDS before every read of LDS.  Who reads waits with wait_loads().
// m0 is named for the compiler's own writes to it; no value lives there, which is what its warning is about.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void load_to_lds(u32x4 base, uint32_t offset, uint32_t k, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "s"(lds), "v"(offset), "s"(base), "s"(k) : "m0", "memory");
}
#pragma clang diagnostic pop
// Until all but the wavefront's last `left` loads are there.
template <int left>
__device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(left) : "memory"); }

// 32 columns from `col` on by 16 rows of a turn's blocks in LDS, as an operand whose rows the columns are: a lane gets eight rows of a
// column.  Sixteen lanes read four rows of sixteen columns, four next to each other each, and are given four rows of one column.
template <bool PAIR>
__device__ inline half8 read_down(const _Float16 *blocks, int across, int h, int col)
{
    typedef short short4v __attribute__((ext_vector_type(4)));
    typedef short short8v __attribute__((ext_vector_type(8)));
    const int lane = threadIdx.x & 63, side = lane / 16 % 2, row = lane / 32 * 8 + lane % 16 / 4, four = lane % 4 * 4;
    const _Float16 *at = PAIR ? blocks + (col / 16 + side) * 512 + row * 32 + h * 16 + four
                              : blocks + (h * across + col / 32) * 512 + row * 32 + side * 16 + four;
    typedef __attribute__((address_space(3))) short4v *lds4;
    const short4v low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)at), high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 4 * 32));
    return __builtin_bit_cast(half8, (short8v)__builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
}

// All wavefronts of the workgroup, each with what it asked of LDS.  (__syncthreads() would wait for the loads to LDS as well.)
__device__ inline void meet()
{
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}

// A buffer of `bytes` from p on, for load_to_lds.
__device__ inline u32x4 buffer_of(const void *p, uint32_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    u32x4 r = {(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, bytes, 0x00027000u};
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (uint32_t)__builtin_amdgcn_readfirstlane((int)r[i]);
    return r;
}

// acc[i][j] += sum over k of P[i][k] Q[j][k] for a wavefront's part of the tile, from rows of K values, over `all` turns from `begin`
// on; rows past the last are others.  Where P and Q are the same rows, they are loaded once.  DOWN: Q is given by columns, as a plane of
// K rows of `across` columns, of which the tile's are those from q_rows on.
// While a turn is multiplied, the next one's values are read from LDS and three more are on their way to it.
template <bool PAIR, bool DOWN, int F>
__device__ __forceinline__ void multiply(const _Float16 *p, const _Float16 *q, uint32_t p_rows, uint32_t q_rows, uint32_t across, uint32_t K, uint32_t begin, uint32_t all, _Float16 *lds,
                                         float16v (&acc)[Form<F>::FI][Form<F>::FJ])
{
    constexpr int T = Form<F>::T, FI = Form<F>::FI, FJ = Form<F>::FJ, W = Form<F>::WI * Form<F>::WJ, KW = Form<F>::KW;
    constexpr int LOADS = 2 * T / 16 / W;   // of 16 rows each, of a wavefront in a turn
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave % W, group = wave / W;
    const int wi = w / Form<F>::WJ * FI * 32, wj = w % Form<F>::WJ * FJ * 32;
    const uint32_t stride = K / kDepth<PAIR> * 1024;   // bytes of 16 rows, a kilobyte a turn
    const uint32_t turns = (all - group + KW - 1) / KW, most = (all + KW - 1) / KW;   // the group's, the first group's
    const bool same = p == q;
    constexpr uint32_t D = kDepth<PAIR>, DEEP = D / 16;      // 16 rows are a block's: of the DEEP ones of a turn, `wide` bytes each
    const uint32_t wide = DOWN ? across / D * 1024 : 0;
    const u32x4 base_p = buffer_of(p, (p_rows < T ? p_rows : T) / 16 * stride), base_q = buffer_of(q, DOWN ? 0 : (q_rows < T ? q_rows : T) / 16 * stride);
    lds += group * kRing * kStage<F>;
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) _Float16 *)lds);
    uint32_t offset[LOADS], to[LOADS];
#pragma unroll
    for (int l = 0; l < LOADS; ++l) {
        const uint32_t first = (w * LOADS + l) * 16;   // of P's T rows, then Q's
        const bool of_q = first >= T;
        const uint32_t rows = of_q ? q_rows : p_rows, r = first % T;   // of which there are a multiple of 64
        offset[l] = (r < rows ? r : rows - 16) / 16 * stride + lane / 4 * 64 + exchanged(lane / 4, lane % 4) * 16;
        if (DOWN && of_q) {   // block r / 16 of the turn's DEEP by T / D, as it is
            const uint32_t at = q_rows / D + r / 16 % (T / D);
            offset[l] = r / 16 / (T / D) * wide + (at < across / D ? at : across / D - 1) * 1024 + lane * 16;
        }
        to[l] = lds0 + first * kTurn * 2;
    }
    const auto fetch = [&](uint32_t turn, int l) __attribute__((always_inline)) {
        const bool of_q = (w * LOADS + l) * 16 >= T;   // a wavefront's loads are of P all, or of Q
        if (of_q && same) return;
        const uint32_t n = begin + turn * KW + group;
        if (DOWN && of_q) load_to_lds(buffer_of(q + (uint64_t)n * DEEP * (wide / 2), DEEP * wide), offset[l], 0, to[l] + turn % kRing * (kStage<F> * 2));
        else load_to_lds(of_q ? base_q : base_p, offset[l], n * 1024, to[l] + turn % kRing * (kStage<F> * 2));
    };
    const auto wait_for = [&](uint32_t turn) {   // after the loads of `turn` up to two more turns' were asked for
        if (turn + 2 < turns) wait_loads<2 * LOADS>();
        else if (turn + 1 < turns) wait_loads<LOADS>();
        else wait_loads<0>();
    };
    half8 a[2][2][FI], b[2][2][FJ];   // of this turn and of the next
    const int q_at = (same ? 0 : T) + wj;
    constexpr int READS = 2 * (FI + FJ), MACS = (PAIR ? 3 : 2) * FI * FJ;
    const auto read = [&](const _Float16 *s, int n, half8 (&av)[2][FI], half8 (&bv)[2][FJ]) __attribute__((always_inline)) {
        const int h = n / (FI + FJ), m = n % (FI + FJ);
        if (DOWN && m < FJ) bv[h][m] = read_down<PAIR>(s + T * kTurn, T / 32, h, wj + m * 32);
        else if (m < FJ) bv[h][m] = *reinterpret_cast<const half8 *>(s + (q_at + m * 32 + lane % 32) * kTurn + exchanged(lane % 32, h * 2 + lane / 32) * 8);
        else av[h][m - FJ] = *reinterpret_cast<const half8 *>(s + (wi + (m - FJ) * 32 + lane % 32) * kTurn + exchanged(lane % 32, h * 2 + lane / 32) * 8);
    };
    const auto mac = [&](int n, const half8 (&av)[2][FI], const half8 (&bv)[2][FJ]) __attribute__((always_inline)) {
        const int g = n / (FI * FJ), i = n % (FI * FJ) / FJ, j = n % FJ;
        const int ha = PAIR ? (g == 1) : g, hb = PAIR ? (g == 0) : g;   // a pair's high parts are [0]: the small products first
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(av[ha][i], bv[hb][j], acc[i][j], 0, 0, 0);
    };
    const auto step = [&](uint32_t t, const half8 (&av)[2][FI], const half8 (&bv)[2][FJ], half8 (&an)[2][FI], half8 (&bn)[2][FJ]) __attribute__((always_inline)) {
        if (t + 1 < turns) wait_for(t + 1);
        meet();                                   // the next turn is there, and all have read this one
        const _Float16 *s = lds + (t + 1) % kRing * kStage<F>;   // behind the last turn: what is left in LDS, unused
#pragma unroll
        for (int l = 0; l < LOADS; ++l) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = READS * l / LOADS; n < READS * (l + 1) / LOADS; ++n) read(s, n, an, bn);
#pragma unroll
            for (int n = MACS * l / LOADS; n < MACS * (l + 1) / LOADS; ++n)
                if (KW == 1 || t < turns) mac(n, av, bv);   // one group: an even number of turns
            if (T > 64) {
#pragma unroll
                for (int n = 0; n < (READS + (DOWN ? 2 * FJ : 0)) / LOADS; ++n) {   // a read behind every product, while there are reads
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (t + 4 < turns) fetch(t + 4, l);
        }
    };
#pragma unroll
    for (uint32_t t = 0; t < kRing; ++t)
#pragma unroll
        for (int l = 0; l < LOADS; ++l)
            if (t < turns) fetch(t, l);
    if (turns > 3) wait_loads<3 * LOADS>();
    else if (turns > 2) wait_loads<2 * LOADS>();
    else if (turns > 1) wait_loads<LOADS>();
    else wait_loads<0>();
    meet();
#pragma unroll
    for (int n = 0; n < READS; ++n) read(lds, n, a[0], b[0]);
    for (uint32_t t = 0; t < most; t += 2) {   // all groups' steps: they meet in every one
        step(t, a[0], b[0], a[1], b[1]);
        step(t + 1, a[1], b[1], a[0], b[0]);
    }
    __syncthreads();
}

// Whether the workgroup is the last of a sum's slices to come, after its stores.  The order of these and of the count is the hardware's, not
// the language's: stores and loads of device scope pass the XCDs' caches by, so what the wait has seen done is where the last one's loads look.
__device__ inline bool last_slice(uint32_t *counter, uint32_t slices, uint32_t *arrived)
{
    wait_loads<0>();   // and stores
    __syncthreads();
    if (threadIdx.x == 0) {
        *arrived = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (*arrived + 1 == slices) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return *arrived + 1 == slices;
}

// One product of every matrix.  A and B are kept without their diagonals, which are fp32: most of a matrix near the identity is
// there, and of its rounding.  With d for A's and e for B's diagonal:
//   B_ij = b A_ij + c ((A A)_ij + (d_i + d_j) A_ij),  e_i = b d_i + c ((A A)_ii + d_i^2),  X <- a X + e hi(X) + B hi(X)
// (the same X in both last terms: an error of X that B as a whole would take out stays taken out).
// `turn`: which of the two X this step reads; it writes the other.
// Which form of a workgroup a launch takes the plan has chosen (choose_tiles): large tiles read least, small ones and slices fill the chip.
template <int OP, bool PAIR, int F>
__global__ __launch_bounds__(kThreads<F>, F == 128 ? 2 : 1) void k_ortho_product(OrthoLayout lay, OrthoCall c, Polynomial f, uint32_t turn)
{
    constexpr int T = Form<F>::T, PL = PAIR ? 2 : 1, WG = kThreads<F>, FI = Form<F>::FI, FJ = Form<F>::FJ;
    // The results go through LDS in blocks of 64 x 64, the groups' sums each: a wavefront's own block, one after the other, or the
    // workgroup's only one.  Its team is the wavefronts that have a part in it.
    constexpr int KW = Form<F>::KW, kTeam = T == 64 ? WG : 64 * KW, kFolds = WG / kTeam * KW, kBlocks = T == 256 ? 2 : 1;
    constexpr size_t kBytes = sizeof(_Float16) * kRing * kStage<F> * KW, kFold = sizeof(float) * kFolds * 64 * kPitch;
    __shared__ __attribute__((aligned(16))) unsigned char lds[kBytes > kFold ? kBytes : kFold];
    __shared__ uint32_t arrived;
    const TileDev t = (OP == GRAM ? lay.gram : OP == SQUARE ? lay.square : lay.product).tiles[blockIdx.x];
    const MatDev &m = lay.mats[t.mat];
    const uint32_t K = OP == GRAM ? m.Np : m.Mp, cols = OP == PRODUCT || OP == LAST ? m.Np : m.Mp;
    const uint64_t plane_x = (uint64_t)m.Mp * m.Np;
    _Float16 *x = c.planes + m.x + turn * 2 * plane_x, *x_next = c.planes + m.x + (turn ^ 1u) * 2 * plane_x;
    _Float16 *a = c.planes + m.a, *b = c.planes + m.b;
    float *diag_a = c.diagonals + m.diag, *diag_b = diag_a + m.Mp;
    const _Float16 *p = OP == GRAM ? x : OP == SQUARE ? a : b;
    const _Float16 *q = OP == GRAM ? x : OP == SQUARE ? a : x;

    const uint32_t lane = threadIdx.x & 63u, w = (threadIdx.x >> 6) % (WG / 64 / KW), group = threadIdx.x / (WG / KW), tid = T == 64 ? threadIdx.x : group * 64 + lane;
    const uint32_t wi = w / Form<F>::WJ * FI * 32, wj = w % Form<F>::WJ * FJ * 32;
    float16v acc[FI][FJ] = {};
    const uint32_t turns = K / kDepth<PAIR>;   // an even number; a slice's too
    const uint32_t begin = turns / 2 * t.slice / t.slices * 2, end = turns / 2 * (t.slice + 1) / t.slices * 2;
    constexpr bool kDown = OP == PRODUCT || OP == LAST;
    multiply<PAIR, kDown, F>(p + (uint64_t)t.i * T * PL * K, kDown ? q : q + (uint64_t)t.j * T * PL * K, m.Mp - t.i * T, kDown ? t.j * T : cols - t.j * T,
                             cols, K, begin, end - begin, reinterpret_cast<_Float16 *>(lds), acc);
    if (T > 64 && t.slices > 1) {
        // The last slice to come adds all of them up, in their order.  The sums pass the caches of the XCDs by (device-scope atomics of
        // 8 bytes; fences would write these caches back): they are where all see them once the wait is over, and counted after that.
        constexpr uint64_t kPlace = KW * T * T / 2;
        uint64_t *sums = reinterpret_cast<uint64_t *>(c.sums) + t.part * kPlace + threadIdx.x;
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    __hip_atomic_store(&sums[t.slice * kPlace + ((i * FJ + j) * 8 + e) * WG],
                                       (uint64_t)__float_as_uint(acc[i][j][e * 2]) | (uint64_t)__float_as_uint(acc[i][j][e * 2 + 1]) << 32,
                                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (!last_slice(c.counters + t.part, t.slices, &arrived)) return;
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) acc[i][j] = float16v{};
        for (uint32_t s = 0; s < t.slices; ++s)
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int j = 0; j < FJ; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint64_t v = __hip_atomic_load(&sums[s * kPlace + ((i * FJ + j) * 8 + e) * WG], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        acc[i][j][e * 2] += __uint_as_float((uint32_t)v);
                        acc[i][j][e * 2 + 1] += __uint_as_float((uint32_t)(v >> 32));
                    }
    }

    float *fold = reinterpret_cast<float *>(lds) + (T == 64 ? 0 : w) * KW * 64 * kPitch, *own = fold + group * 64 * kPitch;
    const bool turned = (OP == LAST && m.tall) || ((OP == GRAM || OP == SQUARE) && t.i != t.j);
    const auto finish = [&](auto which) __attribute__((always_inline)) {
        constexpr int block = decltype(which)::value, BI = FI / kBlocks;
        if (block) __syncthreads();
        const uint32_t in_i = T == 64 ? wi : 0u, in_j = T == 64 ? wj : 0u;   // the wavefront's place in the block
#pragma unroll
        for (int i = 0; i < BI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    own[(in_i + i * 32 + e / 4 * 8 + lane / 32 * 4 + e % 4) * kPitch + in_j + j * 32 + lane % 32] = acc[block * BI + i][j][e];
        __syncthreads();
        bool summed = false;
        if (T == 64 && t.slices > 1) {   // the same with the groups' sums added up first: four elements a thread
            uint64_t *sums = reinterpret_cast<uint64_t *>(c.sums) + (uint64_t)t.part * 2048 + threadIdx.x * 2;
            float *at = fold + threadIdx.x / 16 * kPitch + threadIdx.x % 16 * 4;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = at[e];
#pragma unroll
                for (int g = 1; g < KW; ++g) v[e] += at[g * 64 * kPitch + e];
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
                __hip_atomic_store(&sums[t.slice * 2048 + h], (uint64_t)__float_as_uint(v[h * 2]) | (uint64_t)__float_as_uint(v[h * 2 + 1]) << 32,
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (!last_slice(c.counters + t.part, t.slices, &arrived)) return;
            uint64_t got[kMostSlices][2];
#pragma unroll
            for (uint32_t s = 0; s < kMostSlices; ++s)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (s < t.slices) got[s][h] = __hip_atomic_load(&sums[s * 2048 + h], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = 0.f;
#pragma unroll
            for (uint32_t s = 0; s < kMostSlices; ++s)
                if (s < t.slices)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] += __uint_as_float((uint32_t)(got[s][e / 2] >> e % 2 * 32));
#pragma unroll
            for (int e = 0; e < 4; ++e) at[e] = v[e];
            summed = true;
            __syncthreads();
        }
        const uint32_t i0 = t.i * T + (T == 64 ? 0u : wi + block * 64), j0 = t.j * T + (T == 64 ? 0u : wj);
        const bool there = i0 < m.Mp && j0 < cols;   // the same for all threads of the block
#pragma unroll 2
        for (uint32_t r = there ? tid / 8 : 64u; r < 64; r += kTeam / 8) {
            const uint32_t k = tid % 8 * 8;
            float *at = fold + r * kPitch + k;
            const uint64_t to = place<PAIR>(i0 + r, j0 + k, cols);
            float sum[8], v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sum[e] = at[e];
#pragma unroll
                for (int g = 1; g < KW; ++g) sum[e] += summed ? 0.f : at[g * 64 * kPitch + e];   // the groups' sums, in their order
            }
            half8 hi = {}, lo = {};   // what the result is added to (asked for ahead of the sums it was no faster: 17.2 -> 18.6 us)
            if (OP != GRAM) {
                const _Float16 *old = OP == SQUARE ? a : x;
                hi = *reinterpret_cast<const half8 *>(old + to);
                if (PAIR || OP != SQUARE) lo = *reinterpret_cast<const half8 *>(old + to + (PAIR ? 16 : plane_x));
            }
            const float di = OP == GRAM ? 0.f : (OP == SQUARE ? diag_a : diag_b)[i0 + r] * (1.f / kScaleX);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (OP == GRAM) v[e] = sum[e] * (1.f / kScaleX);
                if (OP == SQUARE) {
                    const bool on = i0 + r == j0 + k + e;
                    const float d = diag_a[j0 + k + e], aij = on ? d : (float)hi[e] + (float)lo[e];
                    v[e] = f.b * aij + f.c * (sum[e] * (1.f / kScaleX) + (on ? di : di + d * (1.f / kScaleX)) * aij);
                }
                if (OP == PRODUCT || OP == LAST)
                    v[e] = f.a * ((float)hi[e] + (float)lo[e]) + (di * (PAIR ? (float)hi[e] + (float)lo[e] : (float)hi[e]) + sum[e] * (1.f / kScaleB));
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
                if (OP != PRODUCT && i0 + r == j0 + k + e) {
                    (OP == GRAM ? diag_a : diag_b)[i0 + r] = v[e];
                    v[e] = 0.f;
                }
                if (OP == SQUARE) v[e] *= kScaleB / kScaleX;
                _Float16 h, l;
                split(v[e], h, l);
                hi[e] = h;
                lo[e] = l;
                const uint32_t both = (uint32_t)__builtin_bit_cast(uint16_t, h) | (uint32_t)__builtin_bit_cast(uint16_t, l) << 16;
                at[e] = __builtin_bit_cast(float, both);
            }
            _Float16 *dst = OP == GRAM ? a : OP == SQUARE ? b : x_next;
            *reinterpret_cast<half8 *>(dst + to) = hi;
            if (PAIR || OP == PRODUCT) *reinterpret_cast<half8 *>(dst + to + (PAIR ? 16 : plane_x)) = lo;
        }
        if (!turned) return;   // the same for the whole workgroup
        __syncthreads();
#pragma unroll 2
        for (uint32_t r = there ? tid / 8 : 64u; r < 64; r += kTeam / 8) {   // column r of the block
            const uint32_t k = tid % 8 * 8;
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
            _Float16 *dst = OP == GRAM ? a : b;
            const uint64_t to = place<PAIR>(j0 + r, i0 + k, m.Mp);
            *reinterpret_cast<half8 *>(dst + to) = hi;
            if (PAIR) *reinterpret_cast<half8 *>(dst + to + 16) = lo;
        }
    };
    finish(std::integral_constant<int, 0>{});
    if constexpr (kBlocks == 2) finish(std::integral_constant<int, 1>{});
}

// ---- the call -----------------------------------------------------------------------------------------------

template <int OP, bool PAIR>
static void product(const OrthoLayout &lay, const OrthoCall &c, const Polynomial &f, uint32_t turn, hipStream_t s)
{
    const LaunchDev &launch = OP == GRAM ? lay.gram : OP == SQUARE ? lay.square : lay.product;
    const uint32_t form = launch.form, n = launch.n;
    ProfScope prof(OP == GRAM ? K_ORTHO_GRAM : OP == SQUARE ? K_ORTHO_SQUARE : K_ORTHO_PRODUCT, s);
    if (form == 256) k_ortho_product<OP, PAIR, 256><<<dim3(n), dim3(kThreads<256>), 0, s>>>(lay, c, f, turn);
    else if (form == 128) k_ortho_product<OP, PAIR, 128><<<dim3(n), dim3(kThreads<128>), 0, s>>>(lay, c, f, turn);
    else if (form == kForm128Twice) k_ortho_product<OP, PAIR, kForm128Twice><<<dim3(n), dim3(kThreads<kForm128Twice>), 0, s>>>(lay, c, f, turn);
    else k_ortho_product<OP, PAIR, 64><<<dim3(n), dim3(kThreads<64>), 0, s>>>(lay, c, f, turn);
}

template <typename T, bool MUON, bool PAIR>
static hipError_t iterate(const OrthoLayout &lay, const OrthoCall &c, hipStream_t s)
{
    {
        ProfScope prof(K_ORTHO_NORM, s);
        k_ortho_norm<T, MUON><<<dim3(lay.nparts), dim3(256), 0, s>>>(lay, c);
    }
    if (lay.thin) return launch_orthogonalize_thin(lay, c, s);
    {
        ProfScope prof(K_ORTHO_PACK, s);
        k_ortho_pack<T, MUON, PAIR><<<dim3(lay.pack.n), dim3(256), 0, s>>>(lay, c);
    }
    for (uint32_t k = 0; k < c.steps; ++k) {
        const Polynomial f = {c.coefficients[3 * k], c.coefficients[3 * k + 1], c.coefficients[3 * k + 2]};
        product<GRAM, PAIR>(lay, c, f, k & 1u, s);
        product<SQUARE, PAIR>(lay, c, f, 0, s);
        if (k + 1 < c.steps) product<PRODUCT, PAIR>(lay, c, f, k & 1u, s);
        else product<LAST, PAIR>(lay, c, f, k & 1u, s);
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
    if (lay.small) return launch_orthogonalize_small(lay, c, s);
    return lay.products == CO3_PRODUCTS_PAIR ? iterate_of<true>(lay, c, s) : iterate_of<false>(lay, c, s);
}

}  // namespace co3
