// What the host side and the kernels of the Newton-Schulz iteration share (co3_train.cpp, k_ortho.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "co3.h"

namespace co3 {

// The workspace holds every matrix as X (M x N, M <= N: the transpose of a tall one), padded by zeros to multiples of 64 either way, so
// that the products have no edges.  Planes of fp16, in elements from the workspace's planes on; the low parts lie behind the high ones.
struct MatDev {
    uint64_t offset, ld;        // in the caller's vector
    uint64_t x;                 // X twice, of one step and of the next, hi and lo: [Mp][Np]
    uint64_t a, b;              // A = X X^T and B = b A + c A A: [Mp][Mp]; hi, or hi and lo
                                // k_ortho_thin: x and a are fp32 elements of the workspace's sums, X by strips and, twice, the parts of A
    uint32_t rows, cols;        // as the caller has it
    uint32_t M, N, Mp, Np;
    uint32_t part, nparts;      // its partial sums of squares
    uint64_t diag;              // the diagonals of A and of B, fp32 [2][Mp], from the workspace's diagonals on
    float scale;
    uint32_t tall;              // X is the transpose
};

constexpr uint32_t kMostSlices = 8;    // of a sum: the last one to come reads all

// The forms of a workgroup of the products (k_ortho.hip), by the elements of a tile either way; this one has two groups for 128.
constexpr int kForm128Twice = 129;

// One workgroup's tile of a launch over all matrices, or a slice of its sum: the slices' sums meet in places part .. of the
// workspace, counted at the first one's counter.
struct TileDev {
    uint32_t mat;
    uint16_t i, j;
    uint32_t part;
    uint16_t slice, slices;
};
struct LaunchDev {
    const TileDev *tiles;
    uint32_t n, form;           // tiles; what a workgroup is: 256, 128, kForm128Twice or 64
};
// One workgroup's part of a sum of squares: `lines` lines of `len` elements, from element `at` of the matrix on.
struct PartDev {
    uint32_t mat, lines;
    uint64_t at, len;
};

constexpr uint32_t kBlock = 64;        // what X is padded to, and a tile of the kernel that lays it out, either way

struct OrthoLayout {
    const MatDev *mats;
    const PartDev *parts;
    LaunchDev pack, gram, square, product;    // of X; of A's lower half; of B's lower half; of X
    uint32_t nmat, nparts;
    uint32_t small;                           // all matrices are: a workgroup takes one through all steps (k_ortho_small.hip)
    uint32_t thin;                            // all have few rows: a workgroup takes 128 columns through a step (there too); pack: these strips
    uint32_t slices;                          // counters of slices, and places for their sums
    uint64_t slice_floats;                    // fp32 elements of these
    int32_t type, products;
    uint64_t diagonals;                       // fp32 elements of all diagonals
};

struct OrthoCall {
    const void *g;
    void *out;                 // nullptr: the model is updated
    float *momentum, *model;
    float eta, beta, decay, eps;
    int32_t nesterov;
    uint32_t steps;
    float coefficients[3 * CO3_MAX_NS_STEPS];
    uint64_t *status;
    double *partial;           // device [nparts]
    uint32_t *counters;        // device [slices], zero between products
    float *sums;               // device: what the slices leave for the last one of a tile
    float *diagonals;          // device
    _Float16 *planes;          // device
};
hipError_t launch_orthogonalize(const OrthoLayout &lay, const OrthoCall &c, hipStream_t s);
constexpr uint32_t kSmallM = 64, kSmallN = 128;   // the largest X of launch_orthogonalize_small
hipError_t launch_orthogonalize_small(const OrthoLayout &lay, const OrthoCall &c, hipStream_t s);
hipError_t launch_orthogonalize_thin(const OrthoLayout &lay, const OrthoCall &c, hipStream_t s);   // behind the norms

}  // namespace co3

struct co3_matrix_plan {
    co3::OrthoLayout lay = {};
    void *tables = nullptr;    // device: all of the layout's
    uint64_t elements = 0;
    size_t workspace_bytes = 0;
    int device = 0;
};
