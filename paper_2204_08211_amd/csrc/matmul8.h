// How a product in 8 bits is cut into workgroups (co3_train8.cpp, k_matmul8.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "co3.h"

namespace co3 {

// The forms of a workgroup: tiles of 256, 128 or 64 rows and columns; up to 16 rows by 16 columns.
constexpr uint32_t kFormRows = 16;

struct Matmul8Plan {
    uint32_t m, n, batch;
    uint32_t turns;                       // of 128 of k
    uint32_t form;
    uint32_t tiles_m, tiles_n, tiles;     // of a matrix
    uint32_t slices;                      // of the sums; 0: nothing to add up
    uint32_t part_ld;                     // floats between the rows of a slice's sums in the workspace, a multiple of 4
};

}  // namespace co3
