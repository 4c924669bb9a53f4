// Host side of the training operators declared in include/co3.h: argument checks, the plan of a set of matrices.
#include <algorithm>
#include <cmath>
#include <functional>
#include <iterator>
#include <map>
#include <new>
#include <queue>
#include <utility>
#include <vector>

#include "co3_internal.h"
#include "ortho.h"
#include "tensor_types.h"

using namespace co3;

namespace {

struct DeviceGuard {
    int prev = 0;
    bool switched = false;
    explicit DeviceGuard(int dev)
    {
        if (hipGetDevice(&prev) == hipSuccess && prev != dev) switched = hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard()
    {
        if (switched) (void)hipSetDevice(prev);
    }
};

inline bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline uint32_t up(uint32_t x, uint32_t n) { return (x + n - 1) / n * n; }
inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool valid_type(int32_t t) { return t == CO3_F32 || t == CO3_BF16 || t == CO3_F16; }

constexpr uint32_t kMaxMatrices = 65536, kMaxSide = 1u << 20;
constexpr uint64_t kMostThreads = (1ull << 32) - 1;   // of a launch: workgroups of 1024 threads at most for tiles, of 256 for norms and layout
constexpr uint64_t kMaxTiles = kMostThreads / 1024, kMaxParts = kMostThreads / 256;

inline uint64_t end_of(const co3_matrix &m) { return m.offset + (uint64_t)(m.rows - 1) * m.ld + m.cols; }

// The sum of floor((a i + b) / m) over i < n, modulo 2^64; a, b < 2^41, m <= 2^40, n <= 2^20.
uint64_t sum_of_floors(uint64_t n, uint64_t m, uint64_t a, uint64_t b)
{
    uint64_t sum = 0;
    while (true) {   // as a greatest common divisor is found: the points below a line, counted by rows or by columns
        sum += n * (n - 1) / 2 * (a / m) + n * (b / m);
        a %= m;
        b %= m;
        const uint64_t top = a * n + b;
        if (top < m) return sum;
        n = top / m;
        b = top % m;
        std::swap(a, m);
    }
}

// Whether two matrices share an element: a row of a begins less than a's columns before a row of b, or within it.
bool meet(const co3_matrix &a, const co3_matrix &b)
{
    const int64_t offset = (int64_t)b.offset, last = offset + (int64_t)((b.rows - 1) * b.ld), wide = a.cols;
    const auto first = [&](int64_t at) {   // the first row of a that begins there or behind it
        const int64_t ahead = at - (int64_t)a.offset;
        return ahead <= 0 ? 0 : std::min<uint64_t>(a.rows, ((uint64_t)ahead + a.ld - 1) / a.ld);
    };
    const uint64_t from = first(offset), to = first(last);
    if (first(offset - wide + 1) < from || to < first(last + b.cols)) return true;   // by b's first row, in b's last row
    // In between: rows that begin at q = q0 + a.ld i from b's first element on, with (q + wide - 1) mod b.ld < wide + b.cols - 1.
    const uint64_t n = to - from, near = (uint64_t)wide + b.cols - 1;
    if (n == 0 || near >= b.ld) return n != 0;
    const uint64_t q = (a.offset + from * a.ld - b.offset + wide - 1) % b.ld, by = a.ld % b.ld;
    return n + sum_of_floors(n, b.ld, by, q) - sum_of_floors(n, b.ld, by, q + b.ld - near) != 0;
}

int check_matrices(uint32_t count, const co3_matrix *m)
{
    for (uint32_t k = 0; k < count; ++k) {
        if (m[k].rows == 0 || m[k].cols == 0 || m[k].rows > kMaxSide || m[k].cols > kMaxSide || m[k].ld < m[k].cols || !std::isfinite(m[k].scale))
            return CO3_ERR_ARG;
        if (m[k].ld > (1ull << 40) || m[k].offset > (1ull << 60)) return CO3_ERR_ARG;   // the last element's index fits 64 bits
    }
    // In the order of their first elements, each against those that have not ended there.  Matrices of the same ld are apart where their
    // columns are: every ld has its open ones' columns, one or two pieces each, in order, and ended ones leave as they are met.
    struct Lane {
        std::map<uint64_t, std::pair<uint64_t, uint64_t>> pieces;   // from a column up to another, until that element
        std::vector<uint32_t> open;
    };
    std::map<uint64_t, Lane> lanes;
    std::vector<uint32_t> order(count);
    for (uint32_t k = 0; k < count; ++k) order[k] = k;
    std::sort(order.begin(), order.end(), [&](uint32_t a, uint32_t b) { return m[a].offset < m[b].offset; });
    for (uint32_t k : order) {
        const co3_matrix &c = m[k];
        for (auto at = lanes.begin(); at != lanes.end();) {
            std::vector<uint32_t> &open = at->second.open;
            if (at->first == c.ld) { ++at; continue; }
            open.erase(std::remove_if(open.begin(), open.end(), [&](uint32_t o) { return end_of(m[o]) <= c.offset; }), open.end());
            for (uint32_t o : open)
                if (meet(m[o], c)) return CO3_ERR_ARG;
            at = open.empty() ? lanes.erase(at) : std::next(at);
        }
        Lane &lane = lanes[c.ld];
        const uint64_t col = c.offset % c.ld, end = col + c.cols;
        const std::pair<uint64_t, uint64_t> pieces[2] = {{col, std::min(end, c.ld)}, {0, end > c.ld ? end - c.ld : 0}};
        for (const auto &[from, to] : pieces) {
            if (from == to) continue;
            auto at = lane.pieces.lower_bound(from);
            if (at != lane.pieces.begin() && std::prev(at)->second.first > from) --at;
            while (at != lane.pieces.end() && at->first < to) {
                if (at->second.second > c.offset) return CO3_ERR_ARG;
                at = lane.pieces.erase(at);
            }
            lane.pieces[from] = {to, end_of(c)};
        }
        lane.open.push_back(k);
    }
    return CO3_OK;
}

// Whether p(s) = a s + b s^3 + c s^5 stays within [-2, 2] and b s^2 + c s^4 within [-7, 7] while s goes from 0 to the largest |p| of
// the step before (1 at first).  Their extremes are at the ends and where p' = a + 3 b t + 5 c t^2 and b + 2 c t vanish, t = s^2.
bool stays_bounded(uint32_t steps, const float *coef)
{
    double top = 1.0;
    for (uint32_t k = 0; k < steps; ++k) {
        const double a = coef[3 * k], b = coef[3 * k + 1], c = coef[3 * k + 2];
        if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
        // p' = 0: one root by the sum of -3 b and the square root that does not cancel, the other from the roots' product a / (5 c), which
        // is -a / (3 b) where c is 0.  NaN and infinities are no place between the ends.
        const double sum = -3 * b - std::copysign(std::sqrt(9 * b * b - 20 * a * c), b);
        const double at[4] = {top * top, -b / (2 * c), sum / (10 * c), 2 * a / sum};
        double most = 0.0, factor = 0.0;
        for (double t : at) {
            if (!(t > 0.0 && t <= top * top)) continue;
            most = std::max(most, std::fabs(std::sqrt(t) * (a + t * (b + t * c))));
            factor = std::max(factor, std::fabs(t * (b + t * c)));
        }
        if (!(most <= 2.0) || !(factor <= 7.0)) return false;
        top = most;
    }
    return true;
}

// What a product of tiles takes, in microseconds, measured with 4096 x 4096 values at a time: a turn of a workgroup (half as deep for
// pairs), what comes before and behind its turns, and how many workgroups the chip has room for.
// What the slices of a sum take to meet, and what the last one takes for each of them, is the last two.
struct Rate { uint32_t form, tile, groups; double turn, pair_turn, ends; uint32_t room; double meet, slice; };
constexpr Rate kRates[] = {{256, 256, 1, 0.96, 1.29, 12.0, 256, 6.0, 4.0},
                           {128, 128, 1, 0.51, 0.67, 8.0, 512, 5.0, 2.0},
                           {kForm128Twice, 128, 2, 0.25, 0.35, 8.0, 256, 5.0, 2.5},
                           {64, 64, 4, 0.12, 0.14, 4.0, 256, 3.5, 0.2}};
constexpr uint32_t kLeastTurns = 16;   // of a slice

enum { GRAM, SQUARE, PRODUCT };
struct Tiles {
    const Rate *rate = nullptr;
    uint32_t parts = 0;
    std::vector<TileDev> v;
};

uint32_t turns_of(const MatDev &m, int op, uint32_t depth) { return (op == GRAM ? m.Np : m.Mp) / depth; }

// Tiles of T x T of a product over all matrices, those with the longest sums first.  Workgroups go to the eight XCDs in turn, each with
// a cache of its own, so every eighth tile is from a neighbourhood: rows of tiles, eight tiles high, are cut into eight pieces.
std::vector<TileDev> tiles_of(const std::vector<MatDev> &mats, int op, uint32_t T, uint32_t depth)
{
    std::vector<uint32_t> order(mats.size());
    for (uint32_t k = 0; k < order.size(); ++k) order[k] = k;
    std::stable_sort(order.begin(), order.end(), [&](uint32_t a, uint32_t b) { return turns_of(mats[a], op, depth) > turns_of(mats[b], op, depth); });
    std::vector<TileDev> out, own;
    for (uint32_t k : order) {
        const uint32_t ni = (mats[k].Mp + T - 1) / T, nj = op != PRODUCT ? ni : (mats[k].Np + T - 1) / T;
        own.clear();
        for (uint32_t i0 = 0; i0 < ni; i0 += 8)
            for (uint32_t j = 0; j < nj; ++j)
                for (uint32_t i = i0; i < std::min(i0 + 8, ni); ++i)
                    if (op == PRODUCT || j <= i) own.push_back({k, (uint16_t)i, (uint16_t)j, 0, 0, 1});
        const size_t n = own.size();
        size_t start[9];
        for (size_t x = 0; x <= 8; ++x) start[x] = n / 8 * x + std::min<size_t>(x, n % 8);
        for (size_t q = 0; q < n; ++q) out.push_back(own[start[q % 8] + q / 8]);
    }
    return out;
}

// The tiles from number `from` on cut into slices of about `share` turns, the longest slices first.
Tiles cut(const std::vector<MatDev> &mats, int op, const Rate &rate, uint32_t depth, const std::vector<TileDev> &v, size_t from, double share)
{
    Tiles out;
    out.rate = &rate;
    out.v.assign(v.begin(), v.begin() + from);
    const auto length = [&](const TileDev &t) { return turns_of(mats[t.mat], op, depth) / t.slices; };
    for (size_t q = from; q < v.size(); ++q) {
        TileDev t = v[q];
        t.slices = (uint16_t)std::max(1.0, std::min((double)kMostSlices, std::round(turns_of(mats[t.mat], op, depth) / std::max(share, (double)kLeastTurns))));
        t.part = out.parts;
        if (t.slices > 1) out.parts += t.slices;
        for (t.slice = 0; t.slice < t.slices; ++t.slice) out.v.push_back(t);
    }
    std::stable_sort(out.v.begin() + from, out.v.end(), [&](const TileDev &a, const TileDev &b) { return length(a) > length(b); });
    return out;
}

// How long a product takes: every workgroup goes where there is room first.
double time_of(const std::vector<MatDev> &mats, int op, uint32_t depth, const Tiles &t)
{
    const Rate &rate = *t.rate;
    const double turn = depth == 16 ? rate.pair_turn : rate.turn;
    std::priority_queue<double, std::vector<double>, std::greater<double>> busy;
    double last = 0.0;
    for (const TileDev &w : t.v) {
        double at = turns_of(mats[w.mat], op, depth) / w.slices * turn + rate.ends;
        if (w.slices > 1) at += rate.meet + w.slices * rate.slice;
        if (busy.size() >= rate.room) { at += busy.top(); busy.pop(); }
        busy.push(at);
        last = std::max(last, at);
    }
    return last;
}

// The tiles with which a product is done first: whole, the ones behind the last full round of workgroups cut so that they fill one, or
// all cut to the length of an even share of the turns, to parts of it, or to the length of the shorter ones.
Tiles choose_tiles(const std::vector<MatDev> &mats, int op, bool pair)
{
    const uint32_t depth = pair ? 16 : 32;
    Tiles best;
    double least = 0.0;
    for (const Rate &rate : kRates) {
        uint64_t count = 0;
        uint32_t longest = 0;
        for (const MatDev &m : mats) {
            const uint64_t ni = (m.Mp + rate.tile - 1) / rate.tile, nj = (m.Np + rate.tile - 1) / rate.tile;
            count += op == PRODUCT ? ni * nj : ni * (ni + 1) / 2;
            longest = std::max(longest, turns_of(m, op, depth));
        }
        if (best.rate && count > 4 * (uint64_t)rate.room) continue;   // fills the chip with larger tiles as well
        if (count > kMaxTiles) return {};
        const std::vector<TileDev> v = tiles_of(mats, op, rate.tile, depth);
        const size_t room = rate.room, whole = v.size() / room * room;
        double all = 0.0, behind = 0.0;
        for (size_t q = 0; q < v.size(); ++q) (q < whole ? all : behind) += turns_of(mats[v[q].mat], op, depth);
        all += behind;
        const auto consider = [&](size_t from, double share) {
            if (from < v.size() && std::max(share, (double)kLeastTurns) * 1.5 > longest) return;   // nothing would be cut
            Tiles t = cut(mats, op, rate, depth, v, from, share);
            const double time = time_of(mats, op, depth, t);
            if (!best.rate || time < least) { least = time; best = std::move(t); }
        };
        consider(v.size(), 0.0);
        consider(whole, behind / room);
        if (v.size() > 4 * room) continue;
        for (double part : {1.0, 0.7, 0.5, 0.35, 0.25}) consider(0, part * all / room);
        uint32_t before = 0;   // no slice longer than a shorter matrix's whole sum
        for (const TileDev &t : v)
            if (const uint32_t n = turns_of(mats[t.mat], op, depth); n != before && (before = n) != longest) consider(0, n);
    }
    return best;
}

uint64_t gram_elements(const MatDev &m) { return m.M > 32 ? 64 * 64 : 32 * 32; }

// Whether k_ortho_thin takes the matrices: while the parts of A that its workgroups read are few.  Its microseconds against those of the
// products by tiles (fp32, five steps): 64 x 1024 56 : 117; 64 of these 163 : 184, 128 of them 305 : 250 (not taken); 64 x 8192 98 : 147,
// 64 x 32768 244 : 267 (192 from high parts; not taken); 16 of 64 x 4096 189 : 178 (not taken); 32 x 32768 98 : 260; 512 of 16 x 512 303 : 388.
bool thin(const std::vector<MatDev> &mats)
{
    double load = 0.0;
    for (const MatDev &m : mats) {
        const double strips = (m.N + kSmallN - 1) / kSmallN;
        if (m.M > kSmallM) return false;
        load += strips * (1.0 + strips / 64) * (double)(gram_elements(m) / 1024);
    }
    return load <= 2400.0;
}

int build_plan(uint32_t count, const co3_matrix *matrices, co3_matrix_plan *p)
{
    OrthoLayout &l = p->lay;
    const uint32_t PL = l.products == CO3_PRODUCTS_PAIR ? 2 : 1;
    std::vector<MatDev> mats(count);
    std::vector<PartDev> parts;
    std::vector<TileDev> pack;
    uint64_t halves = 0, diagonals = 0;
    for (uint32_t k = 0; k < count; ++k) {
        const co3_matrix &c = matrices[k];
        MatDev &m = mats[k];
        m = {};
        m.offset = c.offset; m.ld = c.ld; m.rows = c.rows; m.cols = c.cols; m.scale = c.scale;
        m.tall = c.rows > c.cols ? 1u : 0u;
        m.M = std::min(c.rows, c.cols);
        m.N = std::max(c.rows, c.cols);
        m.Mp = up(m.M, kBlock);
        m.Np = up(m.N, kBlock);
        m.diag = diagonals; diagonals += 2 * m.Mp;
        const uint64_t plane_x = (uint64_t)m.Mp * m.Np, plane_a = (uint64_t)m.Mp * m.Mp;
        m.x = halves; halves += 4 * plane_x;
        m.a = halves; halves += PL * plane_a;
        m.b = halves; halves += PL * plane_a;
        p->elements = std::max(p->elements, end_of(c));
        // parts of about 16384 elements, but at most 512 of a matrix, and 1024 where a line is more than half of one: every workgroup that lays
        // X out adds them up
        const uint64_t n = (uint64_t)c.rows * c.cols, want = std::max<uint64_t>(16384, (n + 511) / 512 + 7 & ~7ull);
        const bool whole = c.ld == c.cols;
        const uint64_t lines = whole ? 1 : c.rows, len = whole ? n : c.cols;
        const uint64_t cut = (len + want - 1) / want, piece = ((len + cut - 1) / cut + 7) & ~7ull, group = std::max<uint64_t>(1, want / len);
        m.part = (uint32_t)parts.size();
        for (uint64_t r = 0; r < lines; r += group)
            for (uint64_t at = 0; at < len; at += piece)
                parts.push_back({k, (uint32_t)std::min(group, lines - r), r * c.ld + at, std::min(piece, len - at)});
        m.nparts = (uint32_t)parts.size() - m.part;
        if (parts.size() > kMaxParts) return CO3_ERR_CAPACITY;
        if (pack.size() + plane_x / (kBlock * kBlock) > kMaxParts) return CO3_ERR_CAPACITY;
        for (uint32_t i = 0; i < m.Mp / kBlock; ++i)
            for (uint32_t j = 0; j < m.Np / kBlock; ++j) pack.push_back({k, (uint16_t)i, (uint16_t)j, 0, 0, 1});
    }
    l.small = 1;
    for (const MatDev &m : mats) l.small &= m.M <= kSmallM && m.N <= kSmallN;
    l.thin = !l.small && thin(mats);
    Tiles gram, square, product;
    if (l.small || l.thin) {
        halves = diagonals = 0;
    } else {
        gram = choose_tiles(mats, GRAM, PL == 2);
        square = choose_tiles(mats, SQUARE, PL == 2);
        product = choose_tiles(mats, PRODUCT, PL == 2);
        if (!gram.rate || !square.rate || !product.rate) return CO3_ERR_CAPACITY;
    }
    if (l.thin) {
        pack.clear();
        for (uint32_t k = 0; k < count; ++k) {
            MatDev &m = mats[k];
            const uint32_t strips = (m.N + kSmallN - 1) / kSmallN;
            for (uint32_t j = 0; j < strips; ++j) pack.push_back({k, 0, (uint16_t)j, 0, 0, 1});
            m.x = l.slice_floats; l.slice_floats += (uint64_t)strips * kSmallM * kSmallN;
            m.a = l.slice_floats; l.slice_floats += (uint64_t)2 * strips * gram_elements(m);
        }
    }
    for (const Tiles *t : {&gram, &square, &product}) {
        if (!t->rate) continue;
        if (t->v.size() > kMaxTiles) return CO3_ERR_CAPACITY;
        l.slices = std::max(l.slices, t->parts);
        l.slice_floats = std::max(l.slice_floats, (uint64_t)t->parts * t->rate->tile * t->rate->tile * t->rate->groups);
    }
    l.nmat = count;
    l.nparts = (uint32_t)parts.size();
    l.diagonals = diagonals;
    p->workspace_bytes = up256(parts.size() * sizeof(double)) + up256(l.slices * sizeof(uint32_t)) + up256(l.slice_floats * sizeof(float)) +
                         up256(diagonals * sizeof(float)) + halves * sizeof(_Float16);

    const size_t at_parts = up256(mats.size() * sizeof(MatDev));
    const std::vector<TileDev> *all[4] = {&pack, &gram.v, &square.v, &product.v};
    size_t at[5] = {at_parts + up256(parts.size() * sizeof(PartDev))};
    for (int k = 0; k < 4; ++k) at[k + 1] = at[k] + up256(all[k]->size() * sizeof(TileDev));
    if (hipMalloc(&p->tables, at[4]) != hipSuccess) return CO3_ERR_HIP;
    unsigned char *d = static_cast<unsigned char *>(p->tables);
    const auto copy = [&](size_t to, const auto &v) {
        return v.empty() || hipMemcpy(d + to, v.data(), v.size() * sizeof(v[0]), hipMemcpyHostToDevice) == hipSuccess;
    };
    if (!copy(0, mats) || !copy(at_parts, parts)) return CO3_ERR_HIP;
    for (int k = 0; k < 4; ++k)
        if (!copy(at[k], *all[k])) return CO3_ERR_HIP;
    l.mats = reinterpret_cast<const MatDev *>(d);
    l.parts = reinterpret_cast<const PartDev *>(d + at_parts);
    const auto launch = [&](int k, const Rate *rate) {
        return LaunchDev{reinterpret_cast<const TileDev *>(d + at[k]), (uint32_t)all[k]->size(), rate ? rate->form : 0u};
    };
    l.pack = launch(0, nullptr);
    l.gram = launch(1, gram.rate);
    l.square = launch(2, square.rate);
    l.product = launch(3, product.rate);
    return CO3_OK;
}

// What both calls check, and the parts of the call that they share.
int check_call(const co3_matrix_plan *plan, uint32_t steps, const float *coefficients, float eps, void *workspace, size_t workspace_bytes,
               uint64_t *status, OrthoCall *c)
{
    if (!coefficients || steps == 0 || steps > CO3_MAX_NS_STEPS || !(eps >= 0.f) || std::isinf(eps) || !stays_bounded(steps, coefficients))
        return CO3_ERR_ARG;
    if (!workspace || !aligned(workspace, 256) || !aligned(status, 8)) return CO3_ERR_ARG;
    if (workspace_bytes < plan->workspace_bytes) return CO3_ERR_CAPACITY;
    c->steps = steps;
    std::copy(coefficients, coefficients + 3 * steps, c->coefficients);
    c->eps = eps;
    c->status = status;
    c->partial = static_cast<double *>(workspace);
    unsigned char *at = static_cast<unsigned char *>(workspace) + up256(plan->lay.nparts * sizeof(double));
    c->counters = reinterpret_cast<uint32_t *>(at);
    at += up256(plan->lay.slices * sizeof(uint32_t));
    c->sums = reinterpret_cast<float *>(at);
    at += up256(plan->lay.slice_floats * sizeof(float));
    c->diagonals = reinterpret_cast<float *>(at);
    c->planes = reinterpret_cast<_Float16 *>(at + up256(plan->lay.diagonals * sizeof(float)));
    return CO3_OK;
}

}  // namespace

extern "C" {

int co3_matrix_plan_create(uint32_t count, const co3_matrix *matrices, int32_t type, int32_t products, co3_matrix_plan **out)
{
    if (!out) return CO3_ERR_ARG;
    *out = nullptr;
    if (!matrices || count == 0 || count > kMaxMatrices || !valid_type(type) ||
        (products != CO3_PRODUCTS_PAIR && products != CO3_PRODUCTS_HIGH))
        return CO3_ERR_ARG;
    co3_matrix_plan *p = nullptr;
    int rc;
    try {
        rc = check_matrices(count, matrices);
        if (rc != CO3_OK) return rc;
        p = new co3_matrix_plan;
        p->lay.type = type;
        p->lay.products = products;
        rc = hipGetDevice(&p->device) == hipSuccess ? build_plan(count, matrices, p) : CO3_ERR_HIP;
    } catch (const std::exception &) {
        rc = CO3_ERR_CAPACITY;
    }
    if (rc != CO3_OK) {
        co3_matrix_plan_destroy(p);
        return rc;
    }
    *out = p;
    return CO3_OK;
}

void co3_matrix_plan_destroy(co3_matrix_plan *plan)
{
    if (!plan) return;
    DeviceGuard guard(plan->device);
    if (plan->tables) (void)hipFree(plan->tables);
    delete plan;
}

size_t co3_matrix_plan_workspace_bytes(const co3_matrix_plan *plan) { return plan ? plan->workspace_bytes : 0; }
uint64_t co3_matrix_plan_elements(const co3_matrix_plan *plan) { return plan ? plan->elements : 0; }

int co3_orthogonalize(const co3_matrix_plan *plan, const co3_orthogonalize_args *a, void *stream)
{
    if (!plan || !a || !a->g || !a->out) return CO3_ERR_ARG;
    const size_t size = type_bytes(plan->lay.type);
    if (!aligned(a->g, size) || !aligned(a->out, size)) return CO3_ERR_ARG;
    OrthoCall c = {};
    if (int rc = check_call(plan, a->steps, a->coefficients, a->eps, a->workspace, a->workspace_bytes, a->status, &c); rc != CO3_OK) return rc;
    c.g = a->g;
    c.out = a->out;
    DeviceGuard guard(plan->device);
    return launch_orthogonalize(plan->lay, c, static_cast<hipStream_t>(stream)) == hipSuccess ? CO3_OK : CO3_ERR_HIP;
}

int co3_muon_update(const co3_matrix_plan *plan, const co3_muon_args *a, void *stream)
{
    if (!plan || !a || !a->g || !a->momentum || !a->model || plan->lay.type != CO3_F32) return CO3_ERR_ARG;
    if (!aligned(a->g, 4) || !aligned(a->momentum, 4) || !aligned(a->model, 4)) return CO3_ERR_ARG;
    if (a->g == a->momentum || a->g == a->model || a->momentum == a->model) return CO3_ERR_ARG;
    if (!std::isfinite(a->eta) || !std::isfinite(a->beta) || !std::isfinite(a->weight_decay)) return CO3_ERR_ARG;
    OrthoCall c = {};
    if (int rc = check_call(plan, a->steps, a->coefficients, a->eps, a->workspace, a->workspace_bytes, a->status, &c); rc != CO3_OK) return rc;
    c.g = a->g;
    c.momentum = a->momentum;
    c.model = a->model;
    c.eta = a->eta;
    c.beta = a->beta;
    c.decay = a->weight_decay;
    c.nesterov = a->nesterov;
    DeviceGuard guard(plan->device);
    return launch_orthogonalize(plan->lay, c, static_cast<hipStream_t>(stream)) == hipSuccess ? CO3_OK : CO3_ERR_HIP;
}

int co3_layernorm(const co3_layernorm_args *a, void *stream)
{
    if (!a || !valid_type(a->type) || a->cols == 0 || a->cols > CO3_MAX_NORM_COLS || a->rows >= (1ull << 31)) return CO3_ERR_ARG;
    if (!(a->eps >= 0.f) || std::isinf(a->eps)) return CO3_ERR_ARG;
    if (a->rows == 0) return CO3_OK;
    const size_t size = type_bytes(a->type);
    if (!a->x || !a->y || !aligned(a->x, size) || !aligned(a->y, size)) return CO3_ERR_ARG;
    if (!aligned(a->weight, 4) || !aligned(a->bias, 4) || !aligned(a->mean, 4) || !aligned(a->rstd, 4)) return CO3_ERR_ARG;
    if (a->x_stride < a->cols || a->y_stride < a->cols || (a->x == a->y && a->x_stride != a->y_stride)) return CO3_ERR_ARG;
    return launch_layernorm(*a, static_cast<hipStream_t>(stream)) == hipSuccess ? CO3_OK : CO3_ERR_HIP;
}

size_t co3_layernorm_backward_workspace_bytes(uint32_t U, uint64_t rows_per_user, uint32_t cols)
{
    return U == 0 || U > 65535u || cols > CO3_MAX_NORM_COLS ? 0 : layernorm_backward_workspace_bytes(U, rows_per_user, cols);
}

int co3_layernorm_backward(const co3_layernorm_backward_args *a, void *stream)
{
    if (!a || !valid_type(a->type) || a->cols == 0 || a->cols > CO3_MAX_NORM_COLS || a->U == 0 || a->U > 65535u) return CO3_ERR_ARG;
    if (a->rows_per_user >= (1ull << 31) || a->U * a->rows_per_user >= (1ull << 31)) return CO3_ERR_ARG;
    const size_t size = type_bytes(a->type);
    const bool grads = a->dweight || a->dbias;
    if (!aligned(a->weight, 4) || !aligned(a->mean, 4) || !aligned(a->rstd, 4) || !aligned(a->dweight, 4) || !aligned(a->dbias, 4)) return CO3_ERR_ARG;
    if (grads && a->U > 1 && a->grad_stride < a->cols) return CO3_ERR_ARG;
    if (a->rows_per_user) {
        if (!a->dy || !a->x || !a->dx || !a->mean || !a->rstd) return CO3_ERR_ARG;
        if (!aligned(a->dy, size) || !aligned(a->x, size) || !aligned(a->dx, size)) return CO3_ERR_ARG;
        if (a->dy_stride < a->cols || a->x_stride < a->cols || a->dx_stride < a->cols) return CO3_ERR_ARG;
        if ((a->dx == a->dy && a->dx_stride != a->dy_stride) || (a->dx == a->x && a->dx_stride != a->x_stride)) return CO3_ERR_ARG;
    } else if (!grads) {
        return CO3_OK;
    }
    const size_t need = grads ? layernorm_backward_workspace_bytes(a->U, a->rows_per_user, a->cols) : 0;
    if (need) {
        if (!a->workspace || !aligned(a->workspace, 16)) return CO3_ERR_ARG;
        if (a->workspace_bytes < need) return CO3_ERR_CAPACITY;
    }
    return launch_layernorm_backward(*a, static_cast<hipStream_t>(stream)) == hipSuccess ? CO3_OK : CO3_ERR_HIP;
}

}  // extern "C"
