// gemm_plan.h -- how a matrix product is divided among blocks (host only).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace hexk {

int device_cus();

namespace gemm {

// One launch: rows `first` .. first + rows - 1 of D in mt x nt tiles.
struct Part {
    int tile;      // 256, 128 or 64 rows and columns
    int first, rows, mt, nt;
    int steps;     // tiles of k
    int splits, per; // parts of the contraction, of so many steps; 0: runs of all tiles'
                     // steps, as many as compute units (256 only)
};
// D[M][N] over K, `planes` 1 or 3 (float32).  gated: N counts the columns of one
// half, a tile has half its columns of each (64: all of each).
struct Plan {
    int M, N, K, planes;
    int64_t Np; // columns of the split sums
    int parts;
    Part part[2];
};

Plan make_plan(int M, int N, int K, bool gated, int planes);
size_t part_bytes(const Plan &p, bool gated);

} // namespace gemm
} // namespace hexk
