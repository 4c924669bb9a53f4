// Host side of the operators in 8 bits and of group norm declared in include/co3.h: argument checks, how a product is cut into workgroups.
#include <algorithm>
#include <cmath>

#include "blocks8.h"
#include "co3_internal.h"
#include "matmul8.h"
#include "tensor_types.h"

using namespace co3;

namespace {

constexpr uint64_t kMostStride = 1ull << 32, kMostBatchStride = 1ull << 46;   // so that the last element's index fits 64 bits

inline bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool valid_type(int32_t t) { return t == CO3_F32 || t == CO3_BF16 || t == CO3_F16; }

// Whether rows of `cols` elements, `stride` apart, of a batch of matrices `batch_stride` apart, lie each by itself: one matrix behind
// the other, or side by side in the same rows.
bool apart(uint64_t rows, uint64_t cols, uint64_t stride, uint64_t batch, uint64_t batch_stride)
{
    if (rows == 0 || batch == 1) return true;
    const uint64_t within = (rows - 1) * stride + cols, across = (batch - 1) * batch_stride + cols;
    return batch_stride >= within || (batch_stride >= cols && stride >= across);
}

}  // namespace

namespace co3 {

bool valid_blocks8(const co3_blocks8 &b)
{
    if (b.cols == 0 || b.cols > CO3_MAX_BLOCKS8_COLS || b.rows >= (1ull << 31) || b.batch == 0 || b.batch > 65535u) return false;
    if (b.ld < b.cols || b.ld % 16 || b.ld > CO3_MAX_BLOCKS8_LD || b.batch_stride % 16 || b.batch_stride > kMostBatchStride) return false;
    if ((b.block_rows != 1 && b.block_rows != 128) || b.scale_ld % 16 || b.scale_ld < block_rows_of(b)) return false;
    if ((uint64_t)block_columns(b) * b.scale_ld >= (1ull << 31) || !aligned(b.values, 16) || !aligned(b.scales, 16)) return false;
    if (b.rows == 0) return true;
    const uint64_t wide = (b.cols + 15ull) & ~15ull;
    return b.values && b.scales && apart(b.rows, wide, b.ld, b.batch, b.batch_stride);
}

}  // namespace co3

namespace {

constexpr uint64_t kMostTiles = 1ull << 22;   // and slices, of a matrix: fewer than 2^32 threads of a launch

// What a product of tiles takes, in microseconds: a turn of a workgroup by itself, and of all that the chip has room for at a time,
// which share the caches; what comes before its turns and behind them; each for results of 16 bits and of fp32.
// Measured (us; two rounds of workgroups and more by `full`, few of them by `alone`): 8192 x 4096 x 4096 bf16 256 118, 128 158; 4 times 4096^3 fp32 448, 494;
// 8 times 500 x 1024 x 1000 bf16 256 20.5, 128 13.9, 64 18.8; 1000 x 517 x 1001 fp32 128 13.9, 64 8.0; 256 x 256 x 4096 bf16 64 12.2, in four slices 9.1.
struct Rate8 { uint32_t form, room; double alone[2], full[2], ends[2]; };
constexpr Rate8 kRates8[] = {{256, 256, {1.30, 1.60}, {1.80, 3.30}, {6.0, 12.0}},
                             {128, 512, {0.65, 0.75}, {1.20, 1.90}, {4.0, 6.0}},
                             {64, 512, {0.28, 0.35}, {0.80, 0.90}, {3.0, 3.5}}};

double time_of(const Rate8 &rate, const Matmul8Plan &p, bool exact)
{
    const double groups = (double)p.tiles * p.slices * p.batch, rounds = std::ceil(groups / rate.room), busy = std::min(1.0, groups / rate.room);
    const double turn = std::max(rate.alone[exact], rate.full[exact] * busy), turns = std::ceil((double)p.turns / p.slices);
    // slices are written and read once more, by a launch of its own
    const double join = p.slices > 1 ? 4.0 + 8.0 * p.slices * p.batch * p.m * (double)p.part_ld / 6e6 : 0.0;
    return rounds * (rate.ends[exact] + turns * turn) + join;
}

// Checks a product and cuts it: CO3_OK and a plan, or what is wrong.
int plan_matmul8(const co3_matmul8_args &a, Matmul8Plan *p)
{
    if (!valid_type(a.type) || !valid_blocks8(a.a) || !valid_blocks8(a.b)) return CO3_ERR_ARG;
    const bool down_a = a.transpose_a != 0, down_b = a.transpose_b == 0;
    const uint64_t m = down_a ? a.a.cols : a.a.rows, n = down_b ? a.b.cols : a.b.rows;
    const uint64_t k = down_a ? a.a.rows : a.a.cols;
    if (k != (down_b ? a.b.rows : a.b.cols)) return CO3_ERR_ARG;
    if ((down_a && a.a.block_rows != 128) || (down_b && a.b.block_rows != 128)) return CO3_ERR_ARG;
    if (a.a.batch != a.b.batch && a.a.batch != 1 && a.b.batch != 1) return CO3_ERR_ARG;
    *p = {};
    p->m = (uint32_t)m;
    p->n = (uint32_t)n;
    p->batch = std::max(a.a.batch, a.b.batch);
    p->turns = (uint32_t)((k + 127) / 128);
    if (m == 0 || n == 0) return CO3_OK;
    p->part_ld = (uint32_t)((n + 3) & ~3ull);
    const auto take = [&](uint32_t form, uint32_t high, uint32_t slices) {
        const uint64_t all = ((m + high - 1) / high) * ((n + form - 1) / form);
        if (all > kMostTiles || all * slices > kMostTiles) return false;
        p->form = form;
        p->tiles_m = (uint32_t)((m + high - 1) / high);
        p->tiles_n = (uint32_t)((n + form - 1) / form);
        p->tiles = (uint32_t)all;
        p->slices = slices;
        return true;
    };
    if (p->turns == 0) return take(256, 256, 0) ? CO3_OK : CO3_ERR_CAPACITY;
    if (m <= 16 && !down_a && !down_b) return take(kFormRows, kFormRows, 1) ? CO3_OK : CO3_ERR_CAPACITY;
    bool found = false;
    double least = 0.0;
    Matmul8Plan best = *p;
    for (const Rate8 &rate : kRates8)
        for (uint32_t slices = 1; slices <= p->turns && slices <= 32; slices += slices < 4 ? 1 : slices / 2) {
            if (!take(rate.form, rate.form, slices)) continue;
            const double time = time_of(rate, *p, a.type == CO3_F32);
            if (!found || time < least) {
                found = true;
                least = time;
                best = *p;
            }
        }
    if (!found) return CO3_ERR_CAPACITY;
    *p = best;
    return CO3_OK;
}

size_t workspace_of(const Matmul8Plan &p)
{
    return p.slices > 1 ? (size_t)p.slices * p.batch * p.m * p.part_ld * sizeof(float) : 0;
}

inline bool valid_activation(int32_t t) { return t == CO3_ACT_NONE || t == CO3_ACT_RELU || t == CO3_ACT_SILU; }
inline bool valid_groups(uint64_t samples, uint64_t pixels, uint32_t channels, uint32_t groups, int32_t type)
{
    if (!valid_type(type) || channels == 0 || channels > CO3_MAX_NORM_COLS || groups == 0 || channels % groups) return false;
    return pixels != 0 && pixels < (1ull << 31) && samples < (1ull << 31) && samples * pixels < (1ull << 31);
}

}  // namespace

extern "C" {

int co3_quantize8(const co3_quantize8_args *a, void *stream)
{
    if (!a || !valid_type(a->type) || !valid_blocks8(a->out) || !aligned(a->status, 8)) return CO3_ERR_ARG;
    if (a->out.rows == 0) return CO3_OK;
    if (!a->x || !aligned(a->x, type_bytes(a->type)) || a->x_stride < a->out.cols || a->x_stride > kMostStride || a->x_batch_stride > kMostBatchStride) return CO3_ERR_ARG;
    return launch_quantize8(*a, static_cast<hipStream_t>(stream)) == hipSuccess ? CO3_OK : CO3_ERR_HIP;
}

int co3_dequantize8(const co3_dequantize8_args *a, void *stream)
{
    if (!a || !valid_type(a->type) || !valid_blocks8(a->x)) return CO3_ERR_ARG;
    if (a->x.rows == 0) return CO3_OK;
    if (!a->out || !aligned(a->out, type_bytes(a->type)) || a->out_stride < a->x.cols || a->out_stride > kMostStride || a->out_batch_stride > kMostBatchStride) return CO3_ERR_ARG;
    if (!apart(a->x.rows, a->x.cols, a->out_stride, a->x.batch, a->out_batch_stride)) return CO3_ERR_ARG;
    return launch_dequantize8(*a, static_cast<hipStream_t>(stream)) == hipSuccess ? CO3_OK : CO3_ERR_HIP;
}

size_t co3_matmul8_workspace_bytes(const co3_matmul8_args *a)
{
    Matmul8Plan p;
    return a && plan_matmul8(*a, &p) == CO3_OK ? workspace_of(p) : 0;
}

int co3_matmul8(const co3_matmul8_args *a, void *stream)
{
    if (!a) return CO3_ERR_ARG;
    Matmul8Plan p;
    if (const int rc = plan_matmul8(*a, &p); rc != CO3_OK) return rc;
    if (p.m == 0 || p.n == 0) return CO3_OK;
    if (!a->out || !aligned(a->out, type_bytes(a->type)) || a->out_stride < p.n || a->out_stride > kMostStride || a->out_batch_stride > kMostBatchStride) return CO3_ERR_ARG;
    if (!apart(p.m, p.n, a->out_stride, p.batch, a->out_batch_stride)) return CO3_ERR_ARG;
    if (const size_t need = workspace_of(p); need) {
        if (!a->workspace || !aligned(a->workspace, 16)) return CO3_ERR_ARG;
        if (a->workspace_bytes < need) return CO3_ERR_CAPACITY;
    }
    return launch_matmul8(*a, p, static_cast<hipStream_t>(stream)) == hipSuccess ? CO3_OK : CO3_ERR_HIP;
}

size_t co3_groupnorm_workspace_bytes(uint64_t samples, uint64_t pixels, uint32_t channels, uint32_t groups, int32_t type)
{
    return valid_groups(samples, pixels, channels, groups, type) ? groupnorm_workspace_bytes(samples, pixels, channels, groups, type) : 0;
}

int co3_groupnorm(const co3_groupnorm_args *a, void *stream)
{
    if (!a || !valid_groups(a->samples, a->pixels, a->channels, a->groups, a->type) || !valid_activation(a->activation)) return CO3_ERR_ARG;
    if (!(a->eps >= 0.f) || std::isinf(a->eps)) return CO3_ERR_ARG;
    if (a->samples == 0) return CO3_OK;
    const size_t size = type_bytes(a->type);
    if (!a->x || !a->y || !aligned(a->x, size) || !aligned(a->y, size)) return CO3_ERR_ARG;
    if (!aligned(a->weight, 4) || !aligned(a->bias, 4) || !aligned(a->mean, 4) || !aligned(a->rstd, 4)) return CO3_ERR_ARG;
    if (a->x_stride < a->channels || a->y_stride < a->channels || a->x_stride > kMostStride || a->y_stride > kMostStride) return CO3_ERR_ARG;
    if (a->x == a->y && a->x_stride != a->y_stride) return CO3_ERR_ARG;
    if (const size_t need = groupnorm_workspace_bytes(a->samples, a->pixels, a->channels, a->groups, a->type); need) {
        if (!a->workspace || !aligned(a->workspace, 16)) return CO3_ERR_ARG;
        if (a->workspace_bytes < need) return CO3_ERR_CAPACITY;
    }
    return launch_groupnorm(*a, static_cast<hipStream_t>(stream)) == hipSuccess ? CO3_OK : CO3_ERR_HIP;
}

size_t co3_groupnorm_backward_workspace_bytes(uint32_t U, uint64_t samples_per_user, uint64_t pixels, uint32_t channels, uint32_t groups, int32_t type)
{
    if (U == 0 || U > 65535u || samples_per_user >= (1ull << 31) || !valid_groups(U * samples_per_user, pixels, channels, groups, type)) return 0;
    return groupnorm_backward_workspace_bytes(U, samples_per_user, pixels, channels, groups, type);
}

int co3_groupnorm_backward(const co3_groupnorm_backward_args *a, void *stream)
{
    if (!a || a->U == 0 || a->U > 65535u || a->samples_per_user >= (1ull << 31) || !valid_activation(a->activation)) return CO3_ERR_ARG;
    const uint64_t samples = a->U * a->samples_per_user;
    if (!valid_groups(samples, a->pixels, a->channels, a->groups, a->type)) return CO3_ERR_ARG;
    const size_t size = type_bytes(a->type);
    const bool grads = a->dweight || a->dbias;
    if (!aligned(a->weight, 4) || !aligned(a->bias, 4) || !aligned(a->mean, 4) || !aligned(a->rstd, 4) || !aligned(a->dweight, 4) || !aligned(a->dbias, 4))
        return CO3_ERR_ARG;
    if (grads && a->U > 1 && (a->grad_stride < a->channels || a->grad_stride > kMostStride)) return CO3_ERR_ARG;
    if (samples) {
        if (!a->dy || !a->dx || !a->mean || !a->rstd || !aligned(a->dy, size) || !aligned(a->dx, size)) return CO3_ERR_ARG;
        if (a->dy_stride < a->channels || a->dx_stride < a->channels || a->dy_stride > kMostStride || a->dx_stride > kMostStride) return CO3_ERR_ARG;
        if (a->dx == a->dy && a->dx_stride != a->dy_stride) return CO3_ERR_ARG;
        if (a->x) {
            if (!aligned(a->x, size) || a->x_stride < a->channels || a->x_stride > kMostStride || (a->dx == a->x && a->dx_stride != a->x_stride)) return CO3_ERR_ARG;
        } else {
            if (!valid_blocks8(a->x8) || a->x8.cols != a->channels || (a->x8.batch != 1 && a->x8.batch != a->U) ||
                a->x8.rows * a->x8.batch != samples * a->pixels)
                return CO3_ERR_ARG;
        }
    } else if (!grads) {
        return CO3_OK;
    }
    const size_t need = groupnorm_backward_workspace_bytes(a->U, a->samples_per_user, a->pixels, a->channels, a->groups, a->type);
    if (need) {
        if (!a->workspace || !aligned(a->workspace, 16)) return CO3_ERR_ARG;
        if (a->workspace_bytes < need) return CO3_ERR_CAPACITY;
    }
    return launch_groupnorm_backward(*a, static_cast<hipStream_t>(stream)) == hipSuccess ? CO3_OK : CO3_ERR_HIP;
}

}  // extern "C"
