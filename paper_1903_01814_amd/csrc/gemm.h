// gemm.h -- the matrix product under the projections and the feed-forward block.
//
//   D[m][n] = sum over k of Q(m, k) P(n, k),    n contiguous in the output
//
// Operands are bfloat16 in memory, with 16-byte aligned rows of whole vectors
// (k_pack.hip lays others out so).  Each is either contiguous in k ("wide": a
// row of memory is one m or n) or contiguous in m or n ("tall": a row of memory
// is one k); the forward takes wide and wide, the data gradient a tall P (the
// weights as they are), the weight gradient tall and tall.  A float32 operand is
// three bfloat16 planes (attn.h, Split), all of a tile in LDS together, and a product
// six products of planes: the large one in sums of its own, so that it is rounded as
// often as a plain one, and each operand read once for three.
//
// A block has BM x BN of D, its NM x NN waves parts of it in 32 x 32 x 16 products
// with P as the rows.  The sums go through LDS once, 32 rows a wave at a time, so
// that epilogues take eight columns at a time and store 16 bytes a lane.
//
// Tiles of KS k go from memory to LDS without passing registers (a wave's load
// fills 1 KB in lane order; the lanes choose what they load, so the 16-byte
// chunks of each row lie permuted by the row's number, and neither form
// of read meets bank conflicts).  Three tiles take turns: while one is multiplied
// the next two are on their way (weight gradient 4096 x 4096 over 8192: 282 -> 238
// us from one tile ahead to two).  The barrier stands before a tile's last step of
// 16 k, whose operands are in registers by then, so the next tile's first operands
// and the loads of a new tile are issued under that step's products.
//
// What bounds it: the matrix cores, by the share of the time that LDS gives them
// operands.  bfloat16: 16384 x 2048 x 2048 123 us (1114 TFLOP/s), its data gradient
// 116 (1181), 4096 x 4096 over 8192 203 (1351); float32 4096 x 4096 x 4096 194 to 221
// TFLOP/s.  Few steps of k are bound by memory instead: 16384 x 512 x 512 in float32
// takes 62 us, of which 37 are steps and the rest the first loads and the stores, which
// all blocks make at the same time.
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
// lambdas of the kernel: one that stays a call keeps all it refers to in memory
#define HEX_INLINE __attribute__((always_inline))
// An operand's tile in LDS, KS k: rows of KS k (wide), or KS rows of 64 m or n, 64
// of them after 64 (tall).  A load of 1 KB is kRows of its rows.
template <bool TALL, int KS> struct Form {
    using Tile = attn::Tile<attn::Bf16, TALL ? 64 : KS, KS>;
    static constexpr int kPitch = Tile::PITCH, kChunks = kPitch / 16, kRows = 64 / kChunks;
};

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
    int steps;       // tiles of k
    // (M: the row behind the tiles' last one)
    int per;         // steps of a split (grid.y splits); 0: the blocks share all
                     // tiles' steps evenly, in runs that end within tiles
    int first;       // row of D that the tiles start at
    int mt, nt;      // tiles of D
    int half;        // gated: rows of P between a gate's row and its partner's
    float *part;     // split sums [split][M - first][Np], null where there is one; of
                     // runs, a tile each: number tile + block
    int64_t Np;
    float *sums;     // split sums over k of Q, [split][M - first]
};

typedef const __attribute__((address_space(1))) void *GlobalPtr;
typedef __attribute__((address_space(3))) void *LdsPtr;

// A wave's part of an operand's tile: B of its m or n, NW waves.
template <bool TALL, int B, int KS, int NW> struct Loader {
    using F = Form<TALL, KS>;
    static constexpr int J = B * KS / 512 / NW; // loads of 1 KB a wave
    static_assert(J * NW * 512 == B * KS, "whole loads");
    // rows of different loads of a lane are permuted alike
    static_assert(TALL || F::kRows * NW % 16 == 0, "one chunk a lane");
    uint32_t at[J];      // byte of the lane's chunk in the operand's rows of the block
    int k[TALL ? J : 1]; // first k of the chunk in the tile

    // wide: row(i) is the operand's row of tile row i, counted from the block's
    // first; tall: the operand has `cols` from there on
    template <typename Row>
    __device__ __forceinline__ void set(int64_t ld, Row row, int cols, int wave, int lane)
    {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int i = F::kRows * (wave + NW * j) + lane / F::kChunks; // row of LDS
            const int r = TALL ? i % KS : i;
            const int c = (lane % F::kChunks) ^ F::Tile::swz(r);
            uint32_t x;
            if constexpr (TALL) {
                const int col = i / KS * 64 + 8 * c;
                x = static_cast<uint32_t>(r) * static_cast<uint32_t>(ld) +
                    (col < cols ? col : 0); // results of columns past the last are not stored
                k[j] = r;
            } else {
                x = static_cast<uint32_t>(row(r)) * static_cast<uint32_t>(ld) + 8 * c;
                k[0] = 8 * c;
            }
            at[j] = 2 * x;
        }
    }
    // Load j of a tile; base: of the block's rows and the tile's k.  As an
    // instruction of its own, so that the compiler does not wait for loads of one
    // buffer where another is read (it did, in one turn of three); meet() in the
    // kernel waits.  A buffer is read behind a meeting only.  m0, which names the place
    // in LDS, is put back: it is the compiler's, which takes no word that a statement
    // changes it.
    __device__ __forceinline__ void load(char *lds, int wave, const char *base, int j) const
    {
        const uint32_t to = static_cast<uint32_t>(
            reinterpret_cast<uintptr_t>((LdsPtr)(lds + 1024 * (wave + NW * j))));
        uint32_t was;
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                     "global_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                     : "=&s"(was)
                     : "s"(to), "v"(at[j]), "s"(base));
    }
    // a tile of `left` k: the chunks past them become zeros, each lane in its place
    __device__ __forceinline__ void load_part(char *lds, int wave, const char *base, int left) const
    {
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (k[TALL ? j : 0] < left)
                load(lds, wave, base, j);
            else
                *reinterpret_cast<uint4 *>(lds + 1024 * (wave + NW * j) + 16 * (threadIdx.x & 63)) =
                    uint4{0, 0, 0, 0};
    }
};

// A lane's reads of an operand's fragments: tiles of 32 rows from row r0 (a
// multiple of 32, tall and more than one tile: of 64) on.
template <bool TALL, int KS> struct Reader {
    using F = Form<TALL, KS>;
    static constexpr int kSub = KS * F::kPitch; // tall: bytes of 64 m or n
    int a, b;
    __device__ __forceinline__ Reader(int r0, int lane)
    {
        const int h = lane >> 5;
        if constexpr (TALL) {
            // rows 16 s + 8 h + 0 .. 7 of LDS are the k of a wide fragment; the
            // transposing read takes four of them at a time
            const int r = 8 * h + ((lane & 15) >> 2);
            const int c = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), o = 8 * (lane & 1);
            const int sub = (r0 >> 6) * kSub, d = (r0 & 32) << 1;
            a = sub + ((F::Tile::chunk_at(r, c) + o) ^ d);
            b = sub + ((F::Tile::chunk_at(r + 4, c) + o) ^ d);
        } else {
            a = F::Tile::cols_at(r0 + (lane & 31), h);
            b = 0;
        }
    }
    // tile t of 32 rows, step s of 16 k
    __device__ __forceinline__ bf16x8 read(char *lds, int t, int s) const
    {
        if constexpr (TALL) {
            using lp = __attribute__((address_space(3))) shortx4 *;
            const int off = (t >> 1) * kSub + 16 * s * F::kPitch, d = (t & 1) << 6;
            const shortx4 lo =
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(lds + off + (a ^ d)));
            const shortx4 hi =
                __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(lds + off + (b ^ d)));
            return __builtin_bit_cast(bf16x8,
                                      __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return *reinterpret_cast<const bf16x8 *>(lds + t * (32 * F::kPitch) + (a ^ (s << 5)));
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
// Epi::kSums: sum(m, v) too, with the sums of Q over k (the gradient of a bias): a
// product of ones by the operands that the first column of tiles reads anyway.
// APART: the epilogue has LDS of its own, and a block goes on to further tiles,
// whose first loads are under way during it.
template <int PL, bool TP, bool TQ, int BM, int BN, int KS, int NM, int NN, bool APART, bool GATED,
          typename Epi>
__global__
__launch_bounds__(64 * NM * NN, PL == 3 && BM == 64 && BN == 128 ? 1 : 2) void gemm_k(Args a,
                                                                                  Epi e)
{
    constexpr int NW = NM * NN, WM = BM / NM, WN = BN / NN, TM = WM / 32, TN = WN / 32;
    // a plane of P, then one of Q, and so on
    constexpr int kBytesP = BN * KS * 2, kPlane = (BM + BN) * KS * 2, kBytes = PL * kPlane;
    constexpr int S = KS / 16;
    constexpr int kSlice = 32 * WN * 4;        // a wave's sums in the epilogue
    constexpr int kFirst = kBytes / kSlice;    // waves that s0 has room for
    __shared__ __align__(1024) char s0[kBytes];
    __shared__ __align__(1024) char s1[kBytes];
    __shared__ __align__(1024) char s2[kBytes];
    __shared__ __align__(1024) char sums[APART ? NW * kSlice : 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % NM, wn = wave / NM;
    const Reader<TP, KS> rp(wn * WN, lane);
    const Reader<TQ, KS> rq(wm * WM, lane);
    const int64_t stepP = TP ? KS * a.P.ld : KS, stepQ = TQ ? KS * a.Q.ld : KS;

    // a tile of D, and the run of its steps that this block has
    int tile, first, tiles, m0, n0;
    int64_t at = 0, last = 0; // runs: of all tiles' steps
    if (APART && a.per == 0) {
        const int64_t all = static_cast<int64_t>(a.mt) * a.nt * a.steps;
        at = blockIdx.x * all / gridDim.x;
        last = (blockIdx.x + 1) * all / gridDim.x;
    }
    tile = static_cast<int>(blockIdx.x) - static_cast<int>(gridDim.x);
    // goes on to the next one, if there is one
    auto advance = [&]() HEX_INLINE {
        if (APART && a.per == 0) {
            if (at >= last)
                return false;
            tile = static_cast<int>(at / a.steps);
            first = static_cast<int>(at - static_cast<int64_t>(tile) * a.steps);
            tiles = static_cast<int>(min(static_cast<int64_t>(a.steps - first), last - at));
            at += tiles;
        } else {
            tile += gridDim.x;
            if (tile >= a.mt * a.nt)
                return false;
            first = blockIdx.y * a.per;
            tiles = min(a.per, a.steps - first);
        }
        first = __builtin_amdgcn_readfirstlane(first);
        tiles = __builtin_amdgcn_readfirstlane(tiles);
        int tm, tn;
        tile_of(tile, a.mt, a.nt, tm, tn);
        m0 = __builtin_amdgcn_readfirstlane(a.first + tm * BM);
        n0 = __builtin_amdgcn_readfirstlane(tn * (GATED ? BN / 2 : BN));
        return true;
    };
    using LoadP = Loader<TP, BN, KS, NW>;
    using LoadQ = Loader<TQ, BM, KS, NW>;
    constexpr int kLoads = PL * (LoadP::J + LoadQ::J); // of a wave and a whole tile
    LoadP lp;
    LoadQ lq;
    const char *baseP, *baseQ;
    int k, ahead; // the next tile of k to load, how many there are yet
    auto start = [&]() HEX_INLINE {
        lp.set(
            a.P.ld,
            [&](int r) HEX_INLINE {
                if constexpr (GATED) {
                    // a wave's columns: WN / 2 of the gate, then their partners
                    const int q = r % WN, f = r / WN * (WN / 2) + q % (WN / 2);
                    return min(f, a.half - 1 - n0) + (q >= WN / 2 ? a.half : 0);
                }
                return min(r, a.P.rows - 1 - n0);
            },
            a.P.rows - n0, wave, lane);
        lq.set(
            a.Q.ld, [&](int r) HEX_INLINE { return min(r, a.Q.rows - 1 - m0); }, a.Q.rows - m0,
            wave, lane);
        baseP = reinterpret_cast<const char *>(a.P.p + (TP ? n0 : n0 * a.P.ld));
        baseQ = reinterpret_cast<const char *>(a.Q.p + (TQ ? m0 : m0 * a.Q.ld));
        k = first;
        ahead = tiles;
    };
    // Loads what there is of the next tile of k.  open: whether that was a whole
    // one, so that the number of its loads is known.
    bool open = false;
    auto load = [&](char *lds) HEX_INLINE {
        open = false;
        if (ahead-- <= 0)
            return;
        const int left = a.K - k * KS;
        open = left >= KS;
#pragma unroll
        for (int l = 0; l < PL; ++l) {
            const char *p = baseP + 2 * (k * stepP + l * a.P.plane);
            const char *q = baseQ + 2 * (k * stepQ + l * a.Q.plane);
            char *to = lds + l * kPlane;
            if (open) {
#pragma unroll
                for (int j = 0; j < LoadP::J; ++j)
                    lp.load(to, wave, p, j);
#pragma unroll
                for (int j = 0; j < LoadQ::J; ++j)
                    lq.load(to + kBytesP, wave, q, j);
            } else {
                lp.load_part(to, wave, p, left);
                lq.load_part(to + kBytesP, wave, q, left);
            }
        }
        ++k;
    };
    // Every wave has read what it read of LDS, and its loads are there but for
    // those of the last tile (all, where their number is not known).
    auto meet_open = [&]() HEX_INLINE {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLoads) : "memory");
    };
    auto meet = [&](bool all) HEX_INLINE {
        if (open && !all)
            meet_open();
        else
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };

    constexpr int kSums = PL == 3 ? 2 : 1; // the large products', the small ones'
    floatx16 acc[kSums][TN][TM];
    bf16x8 fp[2][PL][TN], fq[2][PL][TM];
    // operand i in the order that multiply_one takes them
    constexpr int kReads = PL * (TN + TM);
    auto read_one = [&](char *lds, int s, int to, int i) HEX_INLINE {
        const int l = i / (TN + TM), x = i % (TN + TM);
        char *from = lds + l * kPlane;
        if (x >= 1 && x <= TM)
            fq[to][l][x - 1] = rq.read(from + kBytesP, x - 1, s);
        else
            fp[to][l][x == 0 ? 0 : x - TM] = rp.read(from, x == 0 ? 0 : x - TM, s);
    };
    auto read = [&](char *lds, int s, int to) HEX_INLINE {
#pragma unroll
        for (int i = 0; i < kReads; ++i)
            read_one(lds, s, to, i);
    };
    // planes of P and Q of product x
    constexpr int kProducts = (PL == 3 ? 6 : 1) * TN * TM;
    auto multiply_one = [&](int from, int i) HEX_INLINE {
        constexpr int kP[6] = {0, 1, 0, 1, 2, 0}, kQ[6] = {0, 0, 1, 1, 0, 2};
        const int x = i / (TN * TM), j = i / TM % TN, m = i % TM;
        floatx16 &c = acc[PL == 3 && x > 0 ? 1 : 0][j][m];
        c = mma(fp[from][kP[x]][j], fq[from][kQ[x]][m], c);
    };
    // the sums of Q over k, by the waves of the first columns
    constexpr bool SUMS = Epi::kSums && !APART;
    floatx16 total[SUMS ? TM : 1];
    bool adding = false;
    auto add_up = [&](int from) HEX_INLINE {
        if constexpr (SUMS) {
            if (adding) {
                const __bf16 one = static_cast<__bf16>(1.f);
                const bf16x8 ones = {one, one, one, one, one, one, one, one};
#pragma unroll
                for (int l = PL - 1; l >= 0; --l)
#pragma unroll
                    for (int i = 0; i < TM; ++i)
                        total[i] = mma(ones, fq[from][l][i], total[i]);
            }
        }
    };
    auto multiply = [&](int from) HEX_INLINE {
#pragma unroll
        for (int i = 0; i < kProducts; ++i)
            multiply_one(from, i);
        add_up(from);
    };
    // a tile in `here`, its first operands in registers; the next in `next` and the
    // one after it on their way
    auto turn = [&](char *here, char *next) HEX_INLINE {
#pragma unroll
        for (int s = 0; s + 1 < S; ++s) {
            read(here, s + 1, (s + 1) & 1);
            multiply(s & 1);
        }
        meet(false);
        read(next, 0, 0); // after the last tile: what lies there, not used
        load(here);
        multiply((S - 1) & 1);
    };
    // The same where the tile to be loaded is whole: no branch, and reads and loads
    // one by one between the products, not in a row before them (256 x 256, 8192 of
    // k: 545 -> 492 us, 8192 of contraction with a tall P: 512 -> 454).
    auto steady = [&](char *here, char *next) HEX_INLINE {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const bool last = s == S - 1;
            const char *p = baseP + 2 * k * stepP, *q = baseQ + 2 * k * stepQ;
            if (last) {
                meet_open();
                ++k;
                --ahead;
            }
#pragma unroll
            for (int i = 0; i < kProducts; ++i) {
                multiply_one(s & 1, i);
#pragma unroll
                for (int x = 0; x < kReads; ++x)
                    if (x * kProducts / kReads == i)
                        read_one(last ? next : here, last ? 0 : s + 1, (s + 1) & 1, x);
#pragma unroll
                for (int x = 0; x < kLoads; ++x)
                    if (last && x * kProducts / kLoads == i) {
                        constexpr int J = LoadP::J + LoadQ::J;
                        const int l = x / J, j = x % J;
                        char *to = here + l * kPlane;
                        if (j < LoadP::J)
                            lp.load(to, wave, p + 2 * l * a.P.plane, j);
                        else
                            lq.load(to + kBytesP, wave, q + 2 * l * a.Q.plane, j - LoadP::J);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
            add_up(s & 1);
        }
    };
    // Three tiles of k a turn of the loop; one or two before them where they are left
    // over: the first of all goes to ..
    auto begin = [&]() HEX_INLINE {
        if (tiles % 3 == 0)
            load(s0), load(s1);
        else if (tiles % 3 == 1)
            load(s2), load(s0);
        else
            load(s1), load(s2);
    };

    if (!advance())
        return;
    start();
    begin();
    for (bool fresh = false;; fresh = true) {
#pragma unroll
        for (int x = 0; x < kSums; ++x)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i)
                    acc[x][j][i] = floatx16{};
        if constexpr (SUMS) {
            adding = wn == 0 && n0 == 0;
#pragma unroll
            for (int i = 0; i < TM; ++i)
                total[i] = floatx16{};
        }
        meet(fresh); // an epilogue's loads and stores are not counted
        if (tiles % 3 == 0) {
            load(s2);
            read(s0, 0, 0);
        } else if (tiles % 3 == 1) {
            load(s1);
            read(s2, 0, 0);
        } else {
            load(s0);
            read(s1, 0, 0);
            turn(s1, s2);
        }
        if (tiles % 3 != 0)
            turn(s2, s0);
        int t = tiles / 3;
        // all but the last tile of k are whole
#pragma unroll 1
        while (ahead > 3) { // three a time, counted by steady
            steady(s0, s1);
            steady(s1, s2);
            steady(s2, s0);
            --t;
        }
#pragma unroll 1
        for (; t > 0; --t) {
            turn(s0, s1);
            turn(s1, s2);
            turn(s2, s0);
        }
        constexpr int kCols = GATED ? WN / 2 : WN, kLanes = kCols / 8, kRows = 64 / kLanes;
        const int mw = m0 + wm * WM, nw = n0 + wn * kCols;
        const int col = 8 * (lane % kLanes), n = nw + col;
        const bool in = n < a.N;
        // where this lane's split sums go: from row `lead` on, rows `width` apart, the
        // second half of a gated pair `other` behind
        float *part = nullptr;
        int64_t width = (GATED ? 2 : 1) * a.Np, other = a.Np;
        int lead = a.first, limit = a.M;
        if (APART && a.per == 0) {
            if (tiles < a.steps) {
                part = a.part + static_cast<int64_t>(tile + static_cast<int>(blockIdx.x)) * BM * BN +
                       wn * kCols + col;
                width = BN;
                other = BN / 2;
                lead = m0;
                limit = m0 + BM; // all of the tile, whether it is in D or not
            }
        } else if (a.part != nullptr) {
            part = a.part + blockIdx.y * static_cast<int64_t>(a.M - a.first) * width + n;
        }
        const bool store = in || limit != a.M;
        bool on = false;
        __syncthreads();
        if constexpr (APART) {
            on = advance();
            if (on) {
                start();
                begin();
            }
        }

        // A wave's 32 rows of D at a time through LDS, so that a lane has eight
        // columns of a row, neighbouring lanes the next; 16-byte chunks permuted by
        // the row.  A lane's registers 4 r .. 4 r + 3 are columns 8 r + 4 h + 0 .. 3
        // of row lane % 32.
        constexpr int kChunks = WN / 4;
        char *mine = APART           ? sums + wave * kSlice
                     : wave < kFirst ? s0 + wave * kSlice
                                     : s1 + (wave - kFirst) * kSlice;
        const int h = lane >> 5, row = lane & 31;
        if constexpr (SUMS) {
            if (adding && h == 0) {
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const int m = mw + 32 * i + row;
                    if (m >= a.M)
                        continue;
                    if (a.part != nullptr)
                        a.sums[blockIdx.y * static_cast<int64_t>(a.M - a.first) + m - a.first] =
                            total[i][0];
                    else
                        e.sum(m, total[i][0]);
                }
            }
        }
        const auto c = e.cols(in ? n : 0);
        auto chunk = [&](int r, int x) HEX_INLINE {
            return reinterpret_cast<float4 *>(mine +
                                              (r * kChunks + (x ^ (r & (kChunks - 1)))) * 16);
        };
        auto eight = [&](int r, int at, float(&v)[8]) HEX_INLINE {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 f = *chunk(r, at / 4 + i);
                v[4 * i] = f.x, v[4 * i + 1] = f.y, v[4 * i + 2] = f.z, v[4 * i + 3] = f.w;
            }
        };
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int mi = mw + 32 * i;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float v[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        v[x] = PL == 3 ? acc[0][j][i][4 * r + x] + acc[kSums - 1][j][i][4 * r + x]
                                       : acc[0][j][i][4 * r + x];
                    *chunk(row, 8 * j + 2 * r + h) = float4{v[0], v[1], v[2], v[3]};
                }
            __builtin_amdgcn_wave_barrier();
            if (part != nullptr) {
#pragma unroll 1
                for (int r1 = 0; r1 < 32; r1 += kRows) {
                    const int r = r1 + lane / kLanes, m = mi + r;
                    if (m >= limit || !store)
                        continue;
                    float v[8];
                    eight(r, col, v);
                    float *o = part + (m - lead) * width;
                    save_row8<float, true>(o, 8, v);
                    if constexpr (GATED) {
                        eight(r, kCols + col, v);
                        save_row8<float, true>(o + other, 8, v);
                    }
                }
            } else {
                // four rows at a time: their loads together
                constexpr int U = 32 / kRows < 4 ? 32 / kRows : 4;
#pragma unroll 1
                for (int r1 = 0; r1 < 32; r1 += U * kRows) {
                    const int r0 = r1 + lane / kLanes;
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
        if (!on)
            break;
    }
}

// Adds up the splits and does what the product's epilogue would have done;
// a thread takes eight columns.
template <bool GATED, typename Epi>
__global__ __launch_bounds__(kThreads) void join_k(const float *part, const float *sums,
                                                   int splits, int first, int rows, int N,
                                                   int64_t Np, Epi e)
{
    // (fewer than 2^32 threads: the planner's bound of the split sums)
    const uint32_t per = (N + 7) / 8, at = blockIdx.x * kThreads + threadIdx.x;
    const int r = static_cast<int>(at / per), m = first + r, n = static_cast<int>(at % per) * 8;
    if (r >= rows)
        return;
    const int64_t width = (GATED ? 2 : 1) * Np, all = rows * width;
    const float *p = part + r * width + n;
    const auto c = e.cols(n);
    const auto f = e.fetch(m, n);
    float v[8] = {}, u[8] = {}, t = 0.f;
    const bool adds = Epi::kSums && n == 0;
    // W splits' loads go out together: one after another they cost a trip to memory each
    auto add = [&](auto width_of, int s) HEX_INLINE {
        constexpr int W = decltype(width_of)::value;
        float x[W][8], w[GATED ? W : 1][8], y[W];
#pragma unroll
        for (int j = 0; j < W; ++j) {
            row8<float, true>(p + (s + j) * all, 8, x[j]);
            if constexpr (GATED)
                row8<float, true>(p + (s + j) * all + Np, 8, w[j]);
            if constexpr (Epi::kSums)
                y[j] = adds ? sums[(s + j) * static_cast<int64_t>(rows) + r] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < W; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] += x[j][i];
                if constexpr (GATED)
                    u[i] += w[j][i];
            }
            if constexpr (Epi::kSums)
                t += y[j];
        }
    };
    int s = 0;
    for (; s + 8 <= splits; s += 8)
        add(std::integral_constant<int, 8>{}, s);
    if (splits & 4)
        add(std::integral_constant<int, 4>{}, s), s += 4;
    if (splits & 2)
        add(std::integral_constant<int, 2>{}, s), s += 2;
    if (splits & 1)
        add(std::integral_constant<int, 1>{}, s);
    if constexpr (GATED)
        e.done(m, n, v, u, c);
    else
        e.done(m, n, v, c, f);
    if constexpr (Epi::kSums) {
        if (adds)
            e.sum(m, t);
    }
}

// The same for tiles of T x T that several runs share (run b of G: the steps b all /
// G .. of all tiles', one tile after another); whole ones are done.  A block takes
// 256 threads' worth of a tile.
template <int T, bool GATED, typename Epi>
__global__ __launch_bounds__(kThreads) void join_runs_k(Args a, int64_t G, Epi e)
{
    constexpr int kCols = GATED ? T / 2 : T, kItems = T * kCols / 8 / kThreads; // blocks a tile
    const int tile = blockIdx.x / kItems;
    const int item = static_cast<int>(blockIdx.x % kItems) * kThreads + threadIdx.x;
    const int64_t all = static_cast<int64_t>(a.mt) * a.nt * a.steps;
    const int64_t u = static_cast<int64_t>(tile) * a.steps;
    const int64_t b0 = ((u + 1) * G - 1) / all, b1 = ((u + a.steps) * G - 1) / all;
    if (b0 == b1)
        return;
    int tm, tn;
    tile_of(tile, a.mt, a.nt, tm, tn);
    const int r = item / (kCols / 8), c = item % (kCols / 8) * 8;
    const int m = a.first + tm * T + r, n = tn * kCols + c;
    if (m >= a.M || n >= a.N)
        return;
    const auto cols = e.cols(n);
    const auto f = e.fetch(m, n);
    float v[8] = {}, w[8] = {};
    for (int64_t b = b0; b <= b1; ++b) {
        const float *p = a.part + (tile + b) * (T * T) + r * T + c;
        float x[8];
        row8<float, true>(p, 8, x);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] += x[i];
        if constexpr (GATED) {
            row8<float, true>(p + T / 2, 8, x);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                w[i] += x[i];
        }
    }
    if constexpr (GATED)
        e.done(m, n, v, w, cols);
    else
        e.done(m, n, v, cols, f);
}

// Launches a planned product (gemm_plan.h); ws: part_bytes of the plan.
// PL: planes of the operands.
template <int PL, bool TP, bool TQ, bool GATED, typename Epi>
hipError_t launch(const Plan &pl, const Side &P, const Side &Q, int half, float *ws, const Epi &e,
                  hipStream_t st)
{
    hipError_t err = hipSuccess;
    for (int i = 0; i < pl.parts && err == hipSuccess; ++i) {
        const Part &p = pl.part[i];
        Args a;
        a.P = P;
        a.Q = Q;
        a.M = p.first + p.rows;
        a.N = pl.N;
        a.K = pl.K;
        a.steps = p.steps;
        a.per = p.per;
        a.first = p.first;
        a.mt = p.mt;
        a.nt = p.nt;
        a.half = half;
        a.part = p.splits != 1 ? ws : nullptr;
        a.sums = ws + static_cast<int64_t>(p.splits) * p.rows * pl.Np; // part_bytes has room
        a.Np = pl.Np;
        const uint32_t blocks = static_cast<uint32_t>(p.mt * p.nt);
        const dim3 grid(blocks, static_cast<uint32_t>(p.splits));
        if (p.tile == 256) {
            if constexpr (PL == 1) {
                // a block a compute unit, which goes through tiles
                const uint32_t cus = static_cast<uint32_t>(device_cus());
                HEX_LAUNCH((gemm_k<1, TP, TQ, 256, 256, 32, 2, 4, true, GATED, Epi>),
                           dim3(p.splits == 0 || blocks > cus ? cus : blocks), dim3(512), 0, st, a,
                           e);
                if ((err = hipGetLastError()) == hipSuccess && p.splits == 0) {
                    HEX_LAUNCH((join_runs_k<256, GATED, Epi>),
                               dim3(blocks * (256 * 256 / 8 / kThreads / (GATED ? 2 : 1))),
                               dim3(kThreads), 0, st, a, cus, e);
                    err = hipGetLastError();
                }
            }
            continue;
        } else if (p.tile == 128) {
            // float32: twice the waves, which the sums leave registers for
            HEX_LAUNCH((gemm_k<PL, TP, TQ, 128, 128, 32, PL == 3 ? 4 : 2, 2, false, GATED, Epi>),
                       grid, dim3(PL == 3 ? 512 : 256), 0, st, a, e);
        } else {
            HEX_LAUNCH((gemm_k<PL, TP, TQ, 64, GATED ? 128 : 64, PL == 3 ? 32 : 64, 2, 2, false,
                               GATED, Epi>),
                       grid, dim3(256), 0, st, a, e);
        }
        err = hipGetLastError();
        if (err != hipSuccess || p.splits == 1)
            continue;
        const int64_t items = static_cast<int64_t>(p.rows) * ((pl.N + 7) / 8);
        HEX_LAUNCH((join_k<GATED, Epi>),
                   dim3(static_cast<uint32_t>((items + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                   st, static_cast<const float *>(ws), static_cast<const float *>(a.sums), p.splits,
                   p.first, p.rows, pl.N, pl.Np, e);
        err = hipGetLastError();
    }
    return err;
}

} // namespace gemm
} // namespace hexk
