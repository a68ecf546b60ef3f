// gemm_plan.h -- how a matrix product is divided among blocks (host only).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace hexk {

int device_cus();

namespace gemm {

// D[M][N] over K, `planes` 1 or 3 (float32).  gated: N counts the columns of one
// half, a tile has as many of each.
struct Plan {
    int M, N, K;
    int tile;      // rows and columns of a block's tile: 256, 128 or 64
    int mt, nt;    // tiles
    int kt, steps; // tiles of 64 k, and of all products of planes
    int splits, per;
    int64_t Np; // columns of the split sums
};

Plan make_plan(int M, int N, int K, bool gated, int planes);
size_t part_bytes(const Plan &p, bool gated);

} // namespace gemm
} // namespace hexk
