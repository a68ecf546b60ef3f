// gemm_plan.h -- how a matrix product is divided among blocks (host only).
#pragma once

#include <math.h>
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

namespace plan {

// What a tile costs: us a step of k for one block on a compute unit, and for each
// of several; us of a block's start and epilogue.  Fitted to products of 1024 to 16384
// tokens and 1024 to 8192 of k.  Of 18 products of 1027 to 16432 tokens and 104 to 1366
// features the choice is the fastest of all tiles and splits, or within 8 %, but for
// one (4108 x 256 over 683 in float32: 37 us by tiles of 64, 31 by 128 in three
// splits).  What the rule chooses, in us with the packing (float32):
//   16432 x 512 over 512      82 by 128 (and 64 for 48 rows), 89 by 128 alone, 89 by 64
//   512 x 512 over 16432      82 by 128 in 15 splits, 390 in one, 111 by 64 at best
//   1366 x 256 over 4108      43 by 64 in 5 splits, 66 in one, 109 by 128 in one
//   1027 x 216 over 104       9.1 by 64, 13.4 by 128, 10.8 by 64 in two splits
// and in bfloat16:
//   3287 x 200 over 536       5.5 by 64, 8.2 by 128, 10.2 by 64 in two splits
//   51200 x 1024 over 1024 (gelu, residual)  169 by 256 and 64 for the last rows, 178
//                             by 128, 196 by 256 alone, 210 by 256 in runs
//   2048 x 5464 over 16432    385 by 256 in runs, 444 without
struct Tile {
    int planes, rows, cols, ks, per_cu;
    double alone, each, fixed;
};
constexpr Tile kTiles[] = {{1, 256, 256, 32, 1, 0.9, 0.9, 9.0},
                           {1, 128, 128, 32, 3, 0.32, 0.29, 5.0},
                           {1, 64, 64, 64, 3, 0.235, 0.17, 3.0},
                           {3, 128, 128, 32, 1, 1.32, 1.32, 7.0},
                           {3, 64, 64, 32, 2, 0.5, 0.46, 3.0}};

// The unit with the most blocks decides; a split adds its sums' way through
// memory and a launch.
inline double cost(const Part &p, const Tile &t, int64_t Np, bool gated, int cus)
{
    const int64_t blocks = static_cast<int64_t>(p.mt) * p.nt * p.splits;
    const int64_t n = (blocks + cus - 1) / cus;
    const double wide = gated && t.rows == 64 ? 2. : 1.; // 128 columns
    const int64_t rounds = (n + t.per_cu - 1) / t.per_cu;
    double us = wide * p.per * (n == 1 ? t.alone : fmax(t.alone, n * t.each)) + rounds * t.fixed;
    if (p.splits > 1)
        us += 4.0 + 8.0 * p.splits * p.rows * Np * (gated ? 2 : 1) / 4e6;
    return us;
}

// Bytes of split sums.
inline size_t sums(const Part &p, int64_t Np, bool gated)
{
    if (p.splits == 1)
        return 0;
    if (p.splits == 0)
        return (static_cast<size_t>(p.mt) * p.nt + device_cus()) * (256 * 256 * 4);
    // and those of the rows alone
    return static_cast<size_t>(p.splits) * p.rows * (Np * (gated ? 2 : 1) + 1) * 4;
}

// The best of one launch for these rows, by its estimated time.
inline double plan_rows(Part &best, int first, int rows, int N, int K, bool gated, int planes)
{
    double least = 0;
    best = Part{};
    const int cus = device_cus();
    const int64_t Np = (N + 7) / 8 * 8;
    auto offer = [&](const Part &p, double us) {
        if (best.tile == 0 || us < least) {
            least = us;
            best = p;
        }
    };
    for (const Tile &t : kTiles) {
        if (t.planes != planes)
            continue;
        Part p{};
        const int cols = gated && t.rows > 64 ? t.cols / 2 : t.cols;
        p.tile = t.rows;
        p.first = first;
        p.rows = rows;
        p.mt = static_cast<int>((static_cast<int64_t>(rows) + t.rows - 1) / t.rows);
        p.nt = (N + cols - 1) / cols;
        p.steps = (K + t.ks - 1) / t.ks;
        const int64_t blocks = static_cast<int64_t>(p.mt) * p.nt;
        p.splits = 1;
        p.per = p.steps;
        offer(p, cost(p, t, Np, gated, cus));
        if (t.rows == 256) {
            // runs of equal length: at most a few tiles a unit, their sums through memory
            const double units = static_cast<double>(blocks) * p.steps / cus;
            p.splits = 0;
            p.per = 0;
            if (units >= 8 && blocks < 4 * cus)
                offer(p, 0.85 * units + 12.0 + 2.0 * sums(p, Np, gated) / 7e6);
            continue;
        }
        for (int want = 2; want <= 64 && want <= p.steps; want = want < 8 ? want + 1 : want * 5 / 4) {
            p.per = (p.steps + want - 1) / want;
            p.splits = (p.steps + p.per - 1) / p.per;
            if (sums(p, Np, gated) > (size_t{1} << 28) || blocks * p.splits > 4 * cus)
                break;
            if (p.splits > 1)
                offer(p, cost(p, t, Np, gated, cus));
        }
    }
    return least;
}

} // namespace plan

inline Plan make_plan(int M, int N, int K, bool gated, int planes)
{
    using namespace plan;
    Plan pl{};
    pl.M = M;
    pl.N = N;
    pl.K = K;
    pl.planes = planes;
    pl.Np = (N + 7) / 8 * 8;
    pl.parts = 1;
    double least = plan_rows(pl.part[0], 0, M, N, K, gated, planes);
    // as many rows as give every unit the same number of tiles, and the rest by
    // themselves: another launch, 2 us
    const int cus = device_cus();
    for (const Tile &t : kTiles) {
        if (t.planes != planes)
            continue;
        const int cols = gated && t.rows > 64 ? t.cols / 2 : t.cols;
        const int64_t nt = (N + cols - 1) / cols;
        const int64_t mt = (static_cast<int64_t>(M) + t.rows - 1) / t.rows;
        const int64_t each = mt * nt / cus, rows = each * cus / nt * t.rows;
        if (each < 1 || rows < t.rows || rows >= M)
            continue;
        Part a{}, b{};
        a.tile = t.rows;
        a.rows = static_cast<int>(rows);
        a.mt = static_cast<int>(rows / t.rows);
        a.nt = static_cast<int>(nt);
        a.steps = a.per = (K + t.ks - 1) / t.ks;
        a.splits = 1;
        const double us = 2.0 + cost(a, t, pl.Np, gated, cus) +
                          plan_rows(b, a.rows, M - a.rows, N, K, gated, planes);
        if (us < least) {
            least = us;
            pl.parts = 2;
            pl.part[0] = a;
            pl.part[1] = b;
        }
    }
    return pl;
}

// Whether the product can give the sums of its rows' operand beside it: blocks that
// go through tiles do not.
inline bool gives_sums(const Plan &pl)
{
    for (int i = 0; i < pl.parts; ++i)
        if (pl.part[i].tile == 256)
            return false;
    return true;
}

inline size_t part_bytes(const Plan &pl, bool gated)
{
    using plan::sums;
    size_t most = 0;
    for (int i = 0; i < pl.parts; ++i) {
        const size_t n = sums(pl.part[i], pl.Np, gated);
        most = n > most ? n : most;
    }
    return most;
}

} // namespace gemm
} // namespace hexk
