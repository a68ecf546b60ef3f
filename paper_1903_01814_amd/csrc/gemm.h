// gemm.h -- the matrix product under the projections and the feed-forward block.
//
//   D[m][n] = sum over k of Q(m, k) P(n, k),    n contiguous in the output
//
// Operands are bfloat16 in memory, with 16-byte aligned rows of whole vectors
// (k_pack.hip lays others out so).  Each is either contiguous in k ("wide": a
// row of memory is one m or n) or contiguous in m or n ("tall": a row of memory
// is one k); the forward takes wide and wide, the data gradient a tall P (the
// weights as they are), the weight gradient tall and tall.  A float32 operand is
// three bfloat16 planes (attn.h, Split) and a product six products of planes,
// small ones first: the same kernel over six times the contraction.
//
// A block has BM x BN of D, its NM x NN waves parts of it in 32 x 32 x 16 products
// with P as the rows.  The sums go through LDS once, 32 rows a wave at a time, so
// that epilogues take eight columns at a time and store 16 bytes a lane.
//
// Tiles of 64 k go from memory to LDS without passing registers (a wave's load
// fills 1 KB in lane order; the lanes choose what they load, so the 16-byte
// chunks of each 128-byte row lie permuted by the row's number, and neither form
// of read meets bank conflicts).  Two tiles take turns: while one is multiplied
// the next is on its way.  The barrier stands before a tile's last step of 16 k,
// whose operands are in registers by then, so the next tile's first operands and
// the loads of the tile after it are issued under that step's products.
#pragma once

#include "act.h"
#include "attn.h"
#include "gemm_plan.h"

namespace hexk {
namespace gemm {

using attn::bf16x8;
using attn::floatx16;
using attn::mma;
using attn::shortx4;

constexpr int kThreads = 256;
constexpr int kStep = 64;        // k of a tile
constexpr int kPitch = 2 * kStep; // bytes of its rows
using LdsTile = attn::Tile<attn::Bf16, kStep, 64>;

// An operand.  wide: element (r, k) at p + r ld + k, tall: at p + k ld + r; r <
// rows (tall: rows a multiple of 8), k < K of the product (wide: a multiple of
// 8).  Planes lie `plane` elements apart.
struct Side {
    const bf16raw *p;
    int64_t ld, plane;
    int rows;
};

struct Args {
    Side P, Q;
    int M, N, K;
    int kt, steps;   // tiles of k, and of all products of planes
    int per;         // steps of a split (grid.y splits)
    int mt, nt;      // tiles of D
    int half;        // gated: rows of P between a gate's row and its partner's
    float *part;     // split sums [split][M][Np], null where there is one
    int64_t Np;
};

// planes of the six products of a float32 contraction, small ones first: P and
// Q of product i in bits 2 i
constexpr int kPlanesP = 2 | 0 << 2 | 1 << 4 | 1 << 6 | 0 << 8 | 0 << 10;
constexpr int kPlanesQ = 0 | 2 << 2 | 1 << 4 | 0 << 6 | 1 << 8 | 0 << 10;

typedef const __attribute__((address_space(1))) void *GlobalPtr;
typedef __attribute__((address_space(3))) void *LdsPtr;

// A wave's part of an operand's tile: B rows of r in all, NW waves.
template <bool TALL, int B, int NW> struct Loader {
    static constexpr int J = B / 8 / NW; // loads of 1 KB a wave
    uint32_t at[J];                  // byte of the lane's chunk in the operand's rows of the block
    int k[TALL ? J : 1];             // first k of the chunk in the tile

    // wide: row(i) is the operand's row of tile row i, counted from the block's
    // first; tall: the operand has `cols` from there on
    template <typename Row>
    __device__ __forceinline__ Loader(int64_t ld, Row row, int cols, int wave, int lane)
    {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int i = wave + NW * j;
            const int r = 8 * (TALL ? i & 7 : i) + (lane >> 3);
            const int c = (lane & 7) ^ LdsTile::swz(r);
            uint32_t x;
            if constexpr (TALL) {
                const int col = (i >> 3) * 64 + 8 * c;
                x = static_cast<uint32_t>(r) * static_cast<uint32_t>(ld) +
                    (col < cols ? col : 0); // results of columns past the last are not stored
                k[j] = r;
            } else {
                x = static_cast<uint32_t>(row(r)) * static_cast<uint32_t>(ld) + 8 * c;
                k[0] = 8 * c; // for every j: rows 32 apart are permuted alike
            }
            at[j] = 2 * x;
        }
    }
    // base: of the block's rows and the tile's k; left: k that the tile has
    __device__ __forceinline__ void load(char *lds, int wave, const char *base, int left) const
    {
        if (left >= kStep) {
#pragma unroll
            for (int j = 0; j < J; ++j)
                __builtin_amdgcn_global_load_lds((GlobalPtr)(base + at[j]),
                                                 (LdsPtr)(lds + 1024 * (wave + NW * j)), 16, 0, 0);
        } else {
            // chunks past the contraction become zeros, each lane in its place
#pragma unroll
            for (int j = 0; j < J; ++j) {
                char *to = lds + 1024 * (wave + NW * j);
                if (k[TALL ? j : 0] < left)
                    __builtin_amdgcn_global_load_lds((GlobalPtr)(base + at[j]), (LdsPtr)to, 16, 0,
                                                     0);
                else
                    *reinterpret_cast<uint4 *>(to + 16 * (threadIdx.x & 63)) = uint4{0, 0, 0, 0};
            }
        }
    }
};

// A lane's reads of an operand's fragments: T tiles of 32 rows from row r0 (a
// multiple of 32) of a tile on.
template <bool TALL> struct Reader {
    int a, b;
    __device__ __forceinline__ Reader(int r0, int lane)
    {
        const int h = lane >> 5;
        if constexpr (TALL) {
            // rows 16 s + 8 h + 0 .. 7 of LDS are the k of a wide fragment; the
            // transposing read takes four of them at a time
            const int r = 8 * h + ((lane & 15) >> 2);
            const int c = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), o = 8 * (lane & 1);
            const int sub = (r0 >> 6) * (64 * kPitch), d = (r0 & 32) << 1;
            a = sub + ((LdsTile::chunk_at(r, c) + o) ^ d);
            b = sub + ((LdsTile::chunk_at(r + 4, c) + o) ^ d);
        } else {
            a = LdsTile::cols_at(r0 + (lane & 31), h);
            b = 0;
        }
    }
    // tile t of 32 rows, step s of 16 k
    __device__ __forceinline__ bf16x8 read(char *lds, int t, int s) const
    {
        if constexpr (TALL) {
            using lp = __attribute__((address_space(3))) shortx4 *;
            const int off = (t >> 1) * (64 * kPitch) + 16 * s * kPitch, d = (t & 1) << 6;
            const shortx4 lo =
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(lds + off + (a ^ d)));
            const shortx4 hi =
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(lds + off + (b ^ d)));
            return __builtin_bit_cast(bf16x8,
                                      __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return *reinterpret_cast<const bf16x8 *>(lds + t * (32 * kPitch) + (a ^ (s << 5)));
        }
    }
};

// Where block b of a tile grid works: the dies (b mod 8) take runs of tiles, in
// bands of eight rows of tiles, columns within a band one after another, so that
// the tiles a die has at work at a time share rows and columns in its cache.
__device__ __forceinline__ void tile_of(int b, int mt, int nt, int &m, int &n)
{
    const int all = mt * nt, whole = all / 8, rest = all % 8;
    const int die = b % 8, i = b / 8;
    // die d has whole + (d < rest) tiles
    const int t = die * whole + min(die, rest) + i;
    const int band = t / (8 * nt), in = t - band * 8 * nt;
    const int rows = min(8, mt - band * 8);
    n = in / rows;
    m = band * 8 + in % rows;
}

// The product.  Epi is what becomes of the sums, eight columns from n (a
// multiple of 8) of row m at a time:
//   cols(n)          what a column needs, loaded once for all of a lane's rows
//   fetch(m, n)      what an element needs from memory
//   done(m, n, v, cols, fetched)
// GATED: done(m, f, g, u, ..), columns f of both halves.
template <bool TP, bool TQ, int BM, int BN, int NM, int NN, bool GATED, typename Epi>
__global__ __launch_bounds__(64 * NM *NN, 2) void gemm_k(Args a, Epi e)
{
    constexpr int NW = NM * NN, WM = BM / NM, WN = BN / NN, TM = WM / 32, TN = WN / 32;
    constexpr int kBytesP = BN * kPitch, kBytes = (BM + BN) * kPitch;
    __shared__ __align__(1024) char s0[kBytes];
    __shared__ __align__(1024) char s1[kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % NM, wn = wave / NM;
    int tm, tn;
    tile_of(blockIdx.x, a.mt, a.nt, tm, tn);
    const int m0 = tm * BM, n0 = tn * (GATED ? BN / 2 : BN);

    const Loader<TP, BN, NW> lp(
        a.P.ld,
        [&](int r) {
            if constexpr (GATED) {
                // a wave's columns: WN / 2 of the gate, then their partners
                const int q = r % WN, f = r / WN * (WN / 2) + q % (WN / 2);
                return min(f, a.half - 1 - n0) + (q >= WN / 2 ? a.half : 0);
            }
            return min(r, a.P.rows - 1 - n0);
        },
        a.P.rows - n0, wave, lane);
    const Loader<TQ, BM, NW> lq(
        a.Q.ld, [&](int r) { return min(r, a.Q.rows - 1 - m0); }, a.Q.rows - m0, wave, lane);
    const Reader<TP> rp(wn * WN, lane);
    const Reader<TQ> rq(wm * WM, lane);

    const int first = blockIdx.y * a.per, end = min(first + a.per, a.steps);
    const char *baseP = reinterpret_cast<const char *>(a.P.p + (TP ? n0 : n0 * a.P.ld));
    const char *baseQ = reinterpret_cast<const char *>(a.Q.p + (TQ ? m0 : m0 * a.Q.ld));
    // the next tile to load: its product of planes, its k
    int pair = 5, k = first;
    if (a.steps != a.kt) {
        pair = first / a.kt;
        k = first - pair * a.kt;
    }
    auto load = [&](char *lds) {
        const int left = a.K - k * kStep;
        const int64_t k0 = static_cast<int64_t>(k) * kStep;
        const int64_t op = (kPlanesP >> 2 * pair & 3) * a.P.plane + (TP ? k0 * a.P.ld : k0);
        const int64_t oq = (kPlanesQ >> 2 * pair & 3) * a.Q.plane + (TQ ? k0 * a.Q.ld : k0);
        lp.load(lds, wave, baseP + 2 * op, left);
        lq.load(lds + kBytesP, wave, baseQ + 2 * oq, left);
        if (++k == a.kt) {
            k = 0;
            ++pair;
        }
    };

    floatx16 acc[TN][TM] = {};
    bf16x8 fp[2][TN], fq[2][TM];
    auto read = [&](char *lds, int s, int to) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
            fp[to][j] = rp.read(lds, j, s);
#pragma unroll
        for (int i = 0; i < TM; ++i)
            fq[to][i] = rq.read(lds + kBytesP, i, s);
    };
    auto multiply = [&](int from) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i)
                acc[j][i] = mma(fp[from][j], fq[from][i], acc[j][i]);
    };
    // a tile in `here`, its first operands in registers, the next on its way to
    // `next`; more: there is one after that
    auto turn = [&](char *here, char *next, bool more) {
#pragma unroll
        for (int s = 0; s < 3; ++s) {
            read(here, s + 1, (s + 1) & 1);
            multiply(s & 1);
        }
        // every wave has read `here`, and every wave's part of `next` is there
        __syncthreads();
        read(next, 0, 0); // after the last tile: what lies there, not used
        if (more)
            load(here);
        multiply(1);
    };

    // two tiles a turn of the loop; an odd one goes before them
    const int tiles = end - first;
    if (tiles & 1) {
        load(s1);
        __syncthreads();
        if (tiles > 1)
            load(s0);
        read(s1, 0, 0);
        turn(s1, s0, tiles > 2);
    } else {
        load(s0);
        __syncthreads();
        load(s1);
        read(s0, 0, 0);
    }
#pragma unroll 1
    for (int t = tiles & 1; t < tiles; t += 2) {
        turn(s0, s1, t + 2 < tiles);
        turn(s1, s0, t + 3 < tiles);
    }
    __syncthreads();

    // A wave's 32 rows of D at a time through LDS, so that a lane has eight
    // columns of a row, neighbouring lanes the next; 16-byte chunks permuted by
    // the row.  A lane's registers 4 r .. 4 r + 3 are columns 8 r + 4 h + 0 .. 3 of
    // row lane % 32.
    constexpr int kChunks = WN / 4, kSlice = 32 * WN * 4;
    constexpr int kCols = GATED ? WN / 2 : WN, kLanes = kCols / 8, kRows = 64 / kLanes;
    constexpr int kFirst = kBytes / kSlice; // waves that s0 has room for
    char *mine = wave < kFirst ? s0 + wave * kSlice : s1 + (wave - kFirst) * kSlice;
    const int h = lane >> 5, row = lane & 31;
    const int col = 8 * (lane % kLanes), n = n0 + wn * kCols + col;
    const bool in = n < a.N;
    float *part = a.part == nullptr ? nullptr
                                    : a.part + blockIdx.y * static_cast<int64_t>(a.M) *
                                                   (GATED ? 2 : 1) * a.Np + n;
    const auto c = e.cols(in ? n : 0);
    auto chunk = [&](int r, int x) {
        return reinterpret_cast<float4 *>(mine + (r * kChunks + (x ^ (r & (kChunks - 1)))) * 16);
    };
    auto eight = [&](int r, int at, float(&v)[8]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 f = *chunk(r, at / 4 + i);
            v[4 * i] = f.x, v[4 * i + 1] = f.y, v[4 * i + 2] = f.z, v[4 * i + 3] = f.w;
        }
    };
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int mi = m0 + wm * WM + 32 * i;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *chunk(row, 8 * j + 2 * r + h) =
                    float4{acc[j][i][4 * r], acc[j][i][4 * r + 1], acc[j][i][4 * r + 2],
                           acc[j][i][4 * r + 3]};
        __builtin_amdgcn_wave_barrier();
        if (part != nullptr) {
#pragma unroll 1
            for (int r = lane / kLanes; r < 32; r += kRows) {
                const int m = mi + r;
                if (m >= a.M || !in)
                    continue;
                float v[8];
                eight(r, col, v);
                float *o = part + m * ((GATED ? 2 : 1) * a.Np);
                save_row8<float, true>(o, 8, v);
                if constexpr (GATED) {
                    eight(r, kCols + col, v);
                    save_row8<float, true>(o + a.Np, 8, v);
                }
            }
        } else {
            // four rows at a time: their loads together
            constexpr int U = 32 / kRows < 4 ? 32 / kRows : 4;
#pragma unroll 1
            for (int r0 = lane / kLanes; r0 < 32; r0 += U * kRows) {
                typename Epi::Fetched f[U];
#pragma unroll
                for (int x = 0; x < U; ++x) {
                    const int m = mi + r0 + x * kRows;
                    f[x] = e.fetch(m < a.M ? m : 0, in ? n : 0);
                }
#pragma unroll
                for (int x = 0; x < U; ++x) {
                    const int r = r0 + x * kRows, m = mi + r;
                    float v[8];
                    eight(r, col, v);
                    if constexpr (GATED) {
                        float u[8];
                        eight(r, kCols + col, u);
                        if (m < a.M && in)
                            e.done(m, n, v, u, c);
                    } else if (m < a.M && in) {
                        e.done(m, n, v, c, f[x]);
                    }
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Adds up the splits and does what the product's epilogue would have done;
// a thread takes eight columns.
template <bool GATED, typename Epi>
__global__ __launch_bounds__(kThreads) void join_k(const float *part, int splits, int M, int N,
                                                   int64_t Np, Epi e)
{
    const int64_t per = (N + 7) / 8, at = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (at >= M * per)
        return;
    const int m = static_cast<int>(at / per), n = static_cast<int>(at % per) * 8;
    const int64_t width = (GATED ? 2 : 1) * Np, all = M * width;
    const float *p = part + m * width + n;
    const auto c = e.cols(n);
    const auto f = e.fetch(m, n);
    float v[8] = {}, u[8] = {};
    for (int s = 0; s < splits; ++s) {
        float x[8];
        row8<float, true>(p + s * all, 8, x);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] += x[i];
        if constexpr (GATED) {
            row8<float, true>(p + s * all + Np, 8, x);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                u[i] += x[i];
        }
    }
    if constexpr (GATED)
        e.done(m, n, v, u, c);
    else
        e.done(m, n, v, c, f);
}

// Launches a planned product (gemm_plan.h); ws: gemm_part_bytes of the plan.
template <bool TP, bool TQ, bool GATED, typename Epi>
hipError_t launch(const Plan &pl, const Side &P, const Side &Q, int half, float *ws, const Epi &e,
                  hipStream_t st)
{
    Args a;
    a.P = P;
    a.Q = Q;
    a.M = pl.M;
    a.N = pl.N;
    a.K = pl.K;
    a.kt = pl.kt;
    a.steps = pl.steps;
    a.per = pl.per;
    a.mt = pl.mt;
    a.nt = pl.nt;
    a.half = half;
    a.part = pl.splits > 1 ? ws : nullptr;
    a.Np = pl.Np;
    const dim3 grid(static_cast<uint32_t>(pl.mt * pl.nt), static_cast<uint32_t>(pl.splits));
    if (pl.tile == 256)
        HEX_LAUNCH((gemm_k<TP, TQ, 256, 256, 2, 4, GATED, Epi>), grid, dim3(512), 0, st, a, e);
    else if (pl.tile == 128)
        HEX_LAUNCH((gemm_k<TP, TQ, 128, 128, 2, 2, GATED, Epi>), grid, dim3(256), 0, st, a, e);
    else
        HEX_LAUNCH((gemm_k<TP, TQ, 64, GATED ? 128 : 64, 2, 2, GATED, Epi>), grid, dim3(256), 0, st,
                   a, e);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || pl.splits == 1)
        return err;
    const int64_t items = static_cast<int64_t>(pl.M) * ((pl.N + 7) / 8);
    HEX_LAUNCH((join_k<GATED, Epi>), dim3(static_cast<uint32_t>((items + kThreads - 1) / kThreads)),
               dim3(kThreads), 0, st, static_cast<const float *>(ws), pl.splits, pl.M, pl.N, pl.Np,
               e);
    return hipGetLastError();
}

} // namespace gemm
} // namespace hexk
