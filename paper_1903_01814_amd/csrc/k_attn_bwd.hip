// k_attn_bwd.hip -- softmax attention over packed sequences, gradients.
//
// With x, p as in the forward (p made again from q, k and the saved lse) and
// D_i = sum_d do_id o_id:
//   dv_j = sum_i p_ij do_i
//   ds_ij = p_ij (do_i . v_j - D_i)
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i
// Two kernels, each with its sums in registers: attn_dq_k walks the keys for a
// tile of rows (and computes D_i), attn_dkv_k the rows for a tile of keys,
// with all query heads that share the key head among its rows.  The scores
// and do . v are computed twice, 7 products in place of 5; in exchange no sum
// is added up by atomics, each has one order and the result is the same from
// run to run.
//
// Bound by the matrix cores and the vector unit in turn, as the forward, and
// attn_dkv_k by the wait for the next rows as well: neighbouring pieces of a head
// run on all eight dies, each of which fetches the same rows of Q and dO (the
// first batch below: 2419 MB read, 484 once).  24 sequences of 500 to 5000
// tokens, 16 heads of 128 on 4, causal, in bfloat16: dq 850 us (6 of 14 parts of
// the work, 950 TFLOP/s; matrix cores busy 0.43), dk and dv 1340 (810 TFLOP/s;
// 0.35) and 46 to join; 16 of 1027, 8 heads of 64 on 4, in float32: 327, 425 and
// 27 (160, 165 TFLOP/s; 0.45, 0.48).  512 of 20 to 400, 8 heads of 32: 76, 107,
// dq by memory as the forward (394 MB, 5.1 TB/s, 200 once), dk and dv read 360 MB
// where 208 are their tiles' and 133 once.
#include "attn.h"
#include "kernels.h"

namespace hexk {
namespace attn {
namespace {

// ---- how the keys' work is divided.  A tile of keys of one sequence and
// key head takes as many units as it has tiles of rows that see it, and kFixed
// for its own loads and stores.  Causal, a sequence's first keys have the whole
// sequence's rows and its last ones a few, and sequences differ: one block a
// tile left the card idle behind the longest (24 sequences of 500 to 5000
// tokens, 16 heads of 128 on 4: 455 TFLOP/s, against 762 where all are alike).
// So a tile of more than a share, 1 / pl.shares of its head's units (a few
// shares for each block that the card holds at once), is divided evenly among
// its rows.  The list of the pieces, large ones first by classes of size, is
// made by one block of the first kernel; the second's blocks take them off it
// one after another.
// The pieces of a divided tile leave their sums in the workspace, and a third
// kernel adds them up in their order, so that the result does not depend on
// which block took what.  (The last block to end as the one that adds, without
// that kernel: its fences write back and drop a die's whole cache, 1904 -> 2282
// us where many tiles are divided.)
constexpr int kFixed = 4;
// shares of all heads for each block that the card holds (the case above: 1422 us
// and 22 to join with 2, 1375 and 45 with 3, 1341 and 96 with 5)
constexpr int kShares = 3;
constexpr int kClasses = 8; // of pieces by size
constexpr int kLeast = 24;  // units of a share at least: small tiles stay whole

// one sequence's units: k i - a0 is the first row tile that sees key tile i
struct KeyUnits {
    int a0, k, nt, tiles; // nt row tiles, key tiles
    int lo, hi;           // key tiles that all rows see, that any row sees
    __device__ __forceinline__ int first(int i) const
    {
        const int64_t t = static_cast<int64_t>(k) * i - a0;
        return static_cast<int>(t < 0 ? 0 : t < nt ? t : nt);
    }
    // units of the key tiles before j: nt each up to lo, nt + a0 - k i up to hi
    __device__ __forceinline__ int64_t before(int j) const
    {
        const int64_t l = min(lo, j), h = max(min(hi, j), min(lo, j));
        return l * nt + (h - l) * (static_cast<int64_t>(nt) + a0) -
               k * ((l + h - 1) * (h - l) / 2) + static_cast<int64_t>(kFixed) * j;
    }
};

__device__ __forceinline__ KeyUnits key_units(const AttnArgs &a, const KeyPlan &pl, int n, int m)
{
    KeyUnits u;
    u.nt = (n * a.group.G + pl.row_tile - 1) / pl.row_tile;
    u.tiles = static_cast<int>((static_cast<uint32_t>(m) + pl.key_tile - 1) / pl.key_tile);
    u.k = u.a0 = 0;
    u.lo = u.hi = u.tiles;
    if (a.causal) {
        const int64_t x = static_cast<int64_t>(m - n) * a.group.G; // row_tile: a power of two
        u.a0 = static_cast<int>((x + pl.row_tile - 1) >> pl.row_shift);
        u.k = (pl.key_tile >> pl.row_shift) * a.group.G;
        u.lo = u.a0 >= 0 ? u.a0 / u.k + 1 : 0;
        u.hi = u.nt + u.a0 >= 0 ? (u.nt + u.a0) / u.k + 1 : 0;
    }
    return u;
}

struct Sequence {
    int q0, n, k0, m;
};
__device__ __forceinline__ Sequence sequence(const AttnArgs &a, int s)
{
    Sequence r;
    r.q0 = clamp_start(a.q_start, s, a.Tq);
    r.n = max(0, clamp_start(a.q_start, s + 1, a.Tq) - r.q0);
    r.k0 = clamp_start(a.k_start, s, a.Tk);
    r.m = max(0, clamp_start(a.k_start, s + 1, a.Tk) - r.k0);
    return r;
}

// One block of NT threads: the list of pieces of one head (all heads' are
// alike), a thread taking a tile at a time.  lds: plan_lds(NT) bytes.
constexpr int plan_lds(int NT) { return NT * (2 * 8 + kClasses * 4) + (kClasses + 2) * 4; }

template <int NT>
__device__ void make_plan(const AttnArgs &a, const KeyPlan &pl, unsigned char *lds)
{
    int64_t *before = reinterpret_cast<int64_t *>(lds); // units, tiles before each
    int64_t *tbefore = before + NT;                     // thread's run of sequences
    int *counts = reinterpret_cast<int *>(tbefore + NT); // [classes][NT]
    int *ends = counts + NT * kClasses;                   // [classes]; slots, divided tiles
    const int tid = threadIdx.x;
    const int run = (a.S + NT - 1) / NT;
    const int s0 = min(a.S, tid * run), s1 = min(a.S, s0 + run);
    int64_t sum = 0, tiles = 0;
    for (int s = s0; s < s1; ++s) {
        const Sequence q = sequence(a, s);
        const KeyUnits u = key_units(a, pl, q.n, q.m);
        pl.before[s] = static_cast<int>(tiles); // within the run
        sum += u.before(u.tiles);
        tiles += u.tiles;
    }
    before[tid] = sum;
    tbefore[tid] = tiles;
    if (tid < 2)
        ends[kClasses + tid] = 0;
    __syncthreads();
    for (int d = 1; d < NT; d <<= 1) {
        const int64_t v = tid >= d ? before[tid - d] : 0, w = tid >= d ? tbefore[tid - d] : 0;
        __syncthreads();
        before[tid] += v;
        tbefore[tid] += w;
        __syncthreads();
    }
    const int64_t all = before[NT - 1];
    // offsets that do not ascend can ask for more than the list holds: none then
    const int all_tiles =
        tbefore[NT - 1] > pl.room - 2 * pl.shares ? 0 : static_cast<int>(tbefore[NT - 1]);
    __syncthreads();
    tbefore[tid] -= tiles;
    __syncthreads();
    const int64_t share = max((all + pl.shares - 1) / pl.shares, static_cast<int64_t>(kLeast));
    // tile w: its piece (without rows and slot), its rows, its class
    int t0, rows, cls;
    KeyPiece pc;
    auto tile = [&](int w) {
        // the last run, then sequence, whose first tile is not past w
        int c = 0, len = NT;
        while (len > 1) {
            const int half = len >> 1;
            const bool ok = tbefore[c + half] <= w;
            c = ok ? c + half : c;
            len = ok ? len - half : half;
        }
        const int left = w - static_cast<int>(tbefore[c]);
        int s = min(c * run, a.S - 1);
        len = max(1, min(run, a.S - s));
        while (len > 1) {
            const int half = len >> 1;
            const bool ok = pl.before[s + half] <= left;
            s = ok ? s + half : s;
            len = ok ? len - half : half;
        }
        const Sequence q = sequence(a, s);
        const KeyUnits ku = key_units(a, pl, q.n, q.m);
        const int j = left - pl.before[s];
        t0 = ku.first(j);
        rows = ku.nt - t0;
        // divided only where that takes off a fifth and more
        pc.parts = 4 * static_cast<int64_t>(rows + kFixed) <= 5 * share
                       ? 1
                       : static_cast<int>((rows + share - 1) / share);
        pc.q0 = q.q0, pc.n = q.n, pc.k0 = q.k0, pc.m = q.m, pc.key0 = j * pl.key_tile;
        const int64_t size = rows / pc.parts + kFixed; // up to 5/4 of a share
        cls = kClasses - 1 - static_cast<int>(min(6 * size / share, INT64_C(kClasses - 1)));
    };
    // a thread takes tiles that follow one another, and they keep their order
    // within a class: neighbours run at about the same time and read the same
    // rows
    const int each = (all_tiles + NT - 1) / NT;
    const int w0 = min(all_tiles, tid * each), w1 = min(all_tiles, w0 + each);
    for (int c = 0; c < kClasses; ++c)
        counts[c * NT + tid] = 0;
    for (int w = w0; w < w1; ++w) {
        tile(w);
        counts[cls * NT + tid] += pc.parts;
    }
    __syncthreads();
    for (int d = 1; d < NT; d <<= 1) {
        int v[kClasses];
#pragma unroll
        for (int c = 0; c < kClasses; ++c)
            v[c] = tid >= d ? counts[c * NT + tid - d] : 0;
        __syncthreads();
#pragma unroll
        for (int c = 0; c < kClasses; ++c)
            counts[c * NT + tid] += v[c];
        __syncthreads();
    }
    if (tid == 0) {
        *pl.next = pl.blocks; // the first ones are the blocks' own numbers
        int at = 0;
        for (int c = 0; c < kClasses; ++c) {
            at += counts[c * NT + NT - 1];
            ends[c] = pl.ends[c] = at;
        }
    }
    __syncthreads();
    // this thread's next place in each class: counted from the class's end
    for (int c = 0; c < kClasses; ++c) {
        const int last = counts[c * NT + NT - 1];
        const int here = tid > 0 ? counts[c * NT + tid - 1] : 0;
        __syncthreads();
        counts[c * NT + tid] = ends[c] - last + here;
        __syncthreads();
    }
    for (int w = w0; w < w1; ++w) {
        tile(w);
        const int at = counts[cls * NT + tid];
        counts[cls * NT + tid] = at + pc.parts;
        // which slot a piece has decides nothing
        const int slot = pc.parts > 1 ? atomicAdd(ends + kClasses, pc.parts) : 0;
        for (int i = 0; i < pc.parts; ++i) {
            pc.row0 = t0 + static_cast<int>(static_cast<int64_t>(rows) * i / pc.parts);
            pc.row1 = t0 + static_cast<int>(static_cast<int64_t>(rows) * (i + 1) / pc.parts);
            pc.slot = slot + i;
            pl.list[at + i] = pc;
        }
        if (pc.parts > 1) {
            pc.slot = slot;
            pl.divided[atomicAdd(ends + kClasses + 1, 1)] = pc;
        }
    }
    __syncthreads();
    if (tid == 0)
        pl.ends[kClasses] = ends[kClasses + 1];
}

// ---- dq: rows as in the forward, 32 a wave of NW, BK keys a tile.
//   X^T = K Q^T and dP^T = V dO^T (keys as rows), dQ^T += K^T dS^T
// D from a bfloat16 o is off by o's rounding, as much as the sums' own rounding
// where a row sees a few keys and o is as large as v (dq of 8 keys: 3.1e-3
// instead of 2.4e-3).  D is also sum_j p_ij dp_ij, and a row of up to 32 keys
// takes that, from its one tile.
template <typename M, int DC, int BK, int NW, typename E = typename M::E>
__global__ __launch_bounds__(64 * NW, attn_waves(sizeof(E) == 4, DC)) void
attn_dq_k(const E *q, const E *k, const E *v, const E *o, const float *lse, const E *dout, E *dq,
          float *delta, AttnArgs a, AttnGrads gr, KeyPlan pl)
{
    using TL = Tile<M, DC, BK>;
    using Frag = typename M::Frag;
    constexpr int TR = 32 * NW, KT = BK / 32, DT = DC / 32, DS = DC / 16;
    constexpr int TB = TL::SIZE;
    __shared__ __align__(16) unsigned char smem[4 * TB]; // K, V, K, V
    if (blockIdx.x == 0) {
        static_assert(sizeof(smem) >= plan_lds(64 * NW), "");
        make_plan<64 * NW>(a, pl, smem);
        return;
    }

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int h = lane >> 5, col = lane & 31;
    int kvh, w;
    head_and_slot(a, blockIdx.x - 1, kvh, w);
    if (w < 0)
        return;
    const Group g = a.group;
    const Span sp = find_span<TR>(a.q_start, a.S, a.Tq, g.G, w);
    const int rows = sp.n * g.G;
    if (static_cast<int64_t>(sp.tile) * TR >= rows)
        return;
    const int row0 = sp.tile * TR;
    int kb, m;
    key_span(a, sp.seq, sp.begin, sp.n, kb, m);
    const int ahead = m - sp.n;

    const int row = row0 + wave * 32 + col, rc = min(row, rows - 1);
    const int tq = row_token(g, rc), head = kvh * g.G + rc - tq * g.G;
    const int64_t token = sp.begin + tq;
    const int see = row < rows ? (a.causal ? min(m, max(0, tq + ahead + 1)) : m) : 0;
    const E *qp = q + token * a.ldq + head * a.D;
    const E *gp = dout + token * gr.lddo + head * a.D;
    const E *op = o + token * a.ldo + head * a.D;
    const float l = lse[token * a.Hq + head];
    // a row that saw no key: every p is 0
    const Ref ref = l == -HUGE_VALF ? Ref{HUGE_VALF, 0.f} : ref_of_lse(l);
    Frag qf[DS], gf[DS];
    constexpr bool EXACT = sizeof(E) == 2;
    float dl = 0.f;
#pragma unroll
    for (int s = 0; s < DS; ++s) {
        qf[s] = load_frag<M>(qp, 16 * s + 8 * h, a.D);
        gf[s] = load_frag<M>(gp, 16 * s + 8 * h, a.D);
        dl = dot8(gp, op, 16 * s + 8 * h, a.D, dl);
    }
    dl = both_sum(dl);
    const int r_last = min(rows, row0 + TR) - 1;
    const int end = a.causal ? min(m, max(0, row_token(g, r_last) + ahead + 1)) : m;
    const int ntiles = (end + BK - 1) / BK;
    int most = see, least = see;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        most = max(most, __shfl_xor(most, d));
        least = min(least, __shfl_xor(least, d));
    }
    most = __builtin_amdgcn_readfirstlane(most);
    least = __builtin_amdgcn_readfirstlane(least);

    const E *kp = k + kb * a.ldk + kvh * a.D, *vp = v + kb * a.ldv + kvh * a.D;
    Stage<M, DC, BK, 64 * NW> ks, vs;
    const uint32_t ldk = a.ldk * sizeof(E), ldv = a.ldv * sizeof(E);
    // rows past the end repeat the last one: their scores are masked
    auto load = [&](int tile) {
        const int64_t k0 = static_cast<int64_t>(tile) * BK;
        ks.rows(kp + k0 * a.ldk, ldk, m - tile * BK, a.D);
        vs.rows(vp + k0 * a.ldv, ldv, m - tile * BK, a.D);
    };
    auto store = [&](unsigned char *t) {
        ks.put(t);
        vs.put(t + TB);
    };

    int ca = TL::cols_at(col, h);
    typename TL::RowsAt ra = TL::rows_at(lane);
    floatx16 acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
        acc[d] = floatx16{};

    if (ntiles > 0) {
        load(0);
        store(smem);
    }
    __syncthreads();
    for (int j = 0; j < ntiles; ++j) {
        unsigned char *kt = smem + (j & 1) * 2 * TB, *vt = kt + TB;
        const bool more = j + 1 < ntiles;
        in_loop(ca), in_loop(ra.a), in_loop(ra.b);
        if (more)
            load(j + 1);
        if (j * BK < most) {
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                const int key0 = j * BK + 32 * t;
                typename M::Score sc{};
                floatx16 dp = floatx16{};
#pragma unroll
                for (int s = 0; s < DS; ++s) {
                    add_product(TL::read_cols(kt + 32 * t * TL::PITCH, ca, s), qf[s], sc);
                    dp = mma(TL::read_cols(vt + 32 * t * TL::PITCH, ca, s), gf[s], dp);
                }
                floatx16 x = value(sc);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    x[r] = prob<M>(x[r], a, ref.hi, ref.lo);
                if (key0 + 32 > least) {
                    const int left = see - key0 - 4 * h;
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (8 * (r >> 2) + (r & 3) >= left)
                            x[r] = 0.f;
                }
                if (EXACT && t == 0 && j == 0) {
                    float sum = 0.f;
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        sum = fmaf(x[r], dp[r], sum);
                    sum = both_sum(sum);
                    dl = see <= 32 ? sum : dl;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    x[r] *= dp[r] - dl;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const Frag sf = to_frag<M>(x, s);
#pragma unroll
                    for (int d = 0; d < DT; ++d)
                        acc[d] = mma(TL::read_rows(kt, ra, 32 * t + 16 * s, d), sf, acc[d]);
                }
            }
        }
        if (more)
            store(smem + ((j + 1) & 1) * 2 * TB);
        __syncthreads();
    }

    if (row >= rows)
        return;
    if (h == 0)
        delta[token * a.Hq + head] = dl;
    E *p = dq + token * gr.lddq + head * a.D;
#pragma unroll
    for (int d = 0; d < DT; ++d)
        store_col(p, acc[d], 32 * d + 4 * h, a.D, a.scale);
}

// Rows a step of attn_dkv_k takes, as many as the registers hold (64 instead of
// 32: heads of 64 827 -> 687 us, of 80 1359 -> 1200, of 32 117 -> 107, in
// float32 657 -> 613; heads of 128 spill, 1397 -> 1418), and the waves of it that
// a SIMD holds at once.
constexpr int dkv_rows(bool f32, int DC) { return DC <= (f32 ? 32 : 96) ? 64 : 32; }
constexpr int dkv_waves(bool f32, int DC)
{
    return DC <= 32 && !f32 ? 4 : DC <= 64 || !f32 ? 2 : 1;
}

// Tiles of 256 keys instead of 128 (bfloat16, heads past 32) where sequences
// have so many keys on average: half as many reads of Q and dO.  16 heads of
// 128 on 4: 24 sequences of 2048 keys 2010 -> 1730 us, of 500 to 5000 causal
// 1563 -> 1397, 128 of 370 505 -> 471; but 256 of 150 194 -> 228, 512 of 60
// 124 -> 177.  Heads of 64: 24 of 2048 1100 -> 1026, of 500 to 5000 739 -> 687;
// but 128 of 370 263 -> 270, 64 of 470 129 -> 141.
constexpr bool dkv_wide(bool f32, int DC) { return !f32 && DC > 32; }
constexpr int dkv_wide_keys(int DC) { return DC > 96 ? 320 : 1024; }

// ---- dk and dv: tiles of KT keys, 32 a wave; BR rows a step.
//   X = Q K^T and dP = dO V^T (query rows as rows; a lane holds one key),
//   dV^T += dO^T P, dK^T += Q^T dS
// Blocks take pieces off the list until it is empty.
template <typename M, int DC, int BR, int KT, typename E = typename M::E>
__global__ __launch_bounds__(2 * KT, dkv_waves(sizeof(E) == 4, DC)) void
attn_dkv_k(const E *q, const E *k, const E *v, const float *lse, const E *dout, const float *delta,
           E *dk, E *dv, AttnArgs a, AttnGrads gr, KeyPlan pl)
{
    using TL = Tile<M, DC, BR>;
    using VT = Tile<M, DC, KT>;
    constexpr int NT = 2 * KT;
    using Frag = typename M::Frag;
    constexpr int RT = BR / 32, DT = DC / 32, DS = DC / 16;
    constexpr int TB = TL::SIZE;
    static_assert(BR <= 64, "");
    constexpr int BUF = 2 * TB + 4 * BR * 4; // Q, dO; lse, -D, keys seen, lse's rest
    // the values' operands stay in registers where they fit beside the sums
    constexpr bool VL = M::PLANES == 1 && DC > 96;
    __shared__ __align__(16) unsigned char smem[2 * BUF + (VL ? VT::SIZE : 0)];
    __shared__ int next, ends[kClasses];
    unsigned char *vl = smem + 2 * BUF;

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int h = lane >> 5, col = lane & 31;
    const Group g = a.group;
    if (threadIdx.x < kClasses)
        ends[threadIdx.x] = pl.ends[threadIdx.x] * a.Hkv;
    __syncthreads();
    int w = blockIdx.x;
#pragma unroll 1
    while (w < ends[kClasses - 1]) {
        // the number after this one, asked for now and needed at the end
        int after = 0;
        if (threadIdx.x == 0)
            after = atomicAdd(pl.next, 1);
        // class after class, of all heads each
        int c = 0;
        while (w >= ends[c])
            ++c;
        const int first = __builtin_amdgcn_readfirstlane(c > 0 ? ends[c - 1] : 0) / a.Hkv;
        const int of = __builtin_amdgcn_readfirstlane(ends[c]) / a.Hkv - first;
        // heads after one another, or (narrow ones) side by side
        const int i = w - first * a.Hkv, kvh = a.narrow ? i % a.Hkv : i / of;
        const KeyPiece pc = pl.list[first + (a.narrow ? i / a.Hkv : i - kvh * of)];
        const int key0 = pc.key0, m = pc.m, rows = pc.n * g.G, ahead = m - pc.n;
        const int tile0 = pc.row0, ntiles = pc.row1;

        const int key = key0 + wave * 32 + col, kc = min(key, m - 1);
        Frag kf[DS], vf[VL ? 1 : DS];
#pragma unroll
        for (int s = 0; s < DS; ++s) {
            const int64_t at = pc.k0 + kc;
            kf[s] = load_frag<M>(k + at * a.ldk + kvh * a.D, 16 * s + 8 * h, a.D);
            if constexpr (!VL)
                vf[s] = load_frag<M>(v + at * a.ldv + kvh * a.D, 16 * s + 8 * h, a.D);
        }
        if constexpr (VL) {
            Stage<M, DC, KT, NT> vs;
            vs.rows(v + static_cast<int64_t>(pc.k0 + key0) * a.ldv + kvh * a.D,
                    a.ldv * sizeof(E), m - key0, a.D);
            vs.put(vl);
        }

        const E *qp = q + pc.q0 * a.ldq + static_cast<int64_t>(kvh) * g.G * a.D;
        const E *gp = dout + pc.q0 * gr.lddo + static_cast<int64_t>(kvh) * g.G * a.D;
        const float *lp = lse + static_cast<int64_t>(pc.q0) * a.Hq + kvh * g.G;
        const float *dp0 = delta + static_cast<int64_t>(pc.q0) * a.Hq + kvh * g.G;
        Stage<M, DC, BR, NT> qs, gs;
        const uint32_t ldq = a.ldq * sizeof(E), ldg = gr.lddo * sizeof(E);
        const float per_head = 1.f / g.G;
        Ref ls{0.f, 0.f};
        float ds = 0.f;
        int sees = 0;
        auto load = [&](int tile) {
            // rows counted from the tile's first token: x = row, x / G exact
            // in floats (x + 1/2 is at least 1/2 off a multiple of G)
            const int first = row_token(g, tile * BR), skip = tile * BR - first * g.G;
            const int end = skip + rows - 1 - tile * BR;
            const E *qt = qp + first * a.ldq, *gt = gp + first * gr.lddo;
            auto place = [&](int r, int &t, int &hd) {
                const int x = min(skip + r, end);
                t = static_cast<int>((x + 0.5f) * per_head);
                hd = x - __mul24(t, g.G);
            };
#pragma unroll
            for (int i = 0; i < qs.N; ++i) {
                int t, hd;
                place(qs.row(i), t, hd);
                const uint32_t c = __umul24(hd, a.D * sizeof(E)) + qs.place(i);
                qs.get(i, qt, __umul24(t, ldq) + c, a.D);
                gs.get(i, gt, __umul24(t, ldg) + c, a.D);
            }
            if (threadIdx.x < BR) {
                const int r = tile * BR + threadIdx.x;
                int t, hd;
                place(threadIdx.x, t, hd);
                const uint32_t at = (t + first) * a.Hq + hd;
                const float l = lp[at];
                // rows past the end and rows that saw no key: every p is 0
                ls = r >= rows || l == -HUGE_VALF ? Ref{HUGE_VALF, 0.f} : ref_of_lse(l);
                ds = dp0[at];
                sees = r >= rows ? 0 : a.causal ? max(0, t + first + ahead + 1) : m;
            }
        };
        auto store = [&](unsigned char *t) {
            qs.put(t);
            gs.put(t + TB);
            if (threadIdx.x < BR) {
                float *f = reinterpret_cast<float *>(t + 2 * TB);
                f[threadIdx.x] = ls.hi;
                f[BR + threadIdx.x] = -ds;
                reinterpret_cast<int *>(f)[2 * BR + threadIdx.x] = sees;
                f[3 * BR + threadIdx.x] = ls.lo;
            }
        };

        const unsigned char *vw = vl + wave * 32 * TL::PITCH;
        int ca = TL::cols_at(col, h);
        typename TL::RowsAt ra = TL::rows_at(lane);
        floatx16 dka[DT], dva[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d)
            dka[d] = dva[d] = floatx16{};

        if (tile0 < ntiles) {
            load(tile0);
            store(smem);
        }
        __syncthreads();
#pragma unroll 1
        for (int j = tile0; j < ntiles; ++j) {
            unsigned char *qt = smem + ((j - tile0) & 1) * BUF, *gt = qt + TB;
            const float *lt = reinterpret_cast<const float *>(qt + 2 * TB), *dt = lt + BR;
            const int *st = reinterpret_cast<const int *>(dt + BR);
            const bool more = j + 1 < ntiles;
            in_loop(ca), in_loop(ra.a), in_loop(ra.b);
            if (more)
                load(j + 1);
            // the first row of a tile sees the fewest keys, the last (of the
            // rows there are) the most
            const int first_sees = a.causal ? row_token(g, min(j * BR, rows - 1)) + ahead + 1 : m;
            const int last_sees =
                a.causal ? row_token(g, min((j + 1) * BR, rows) - 1) + ahead + 1 : m;
            const int wkey = key0 + wave * 32;
            if (wkey < last_sees) {
                const bool masked = wkey + 32 > first_sees;
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    if (RT > 1 && j * BR + 32 * t >= rows)
                        break;
                    typename M::Score sc{};
                    floatx16 dp; // from -D on
                    const int at = 32 * t + 4 * h;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        set_quad(dp, i, *reinterpret_cast<const float4 *>(dt + at + 8 * i));
#pragma unroll
                    for (int s = 0; s < DS; ++s) {
                        add_product(TL::read_cols(qt + 32 * t * TL::PITCH, ca, s), kf[s], sc);
                        const Frag vs = VL ? VT::read_cols(vw, ca, s) : vf[VL ? 0 : s];
                        dp = mma(TL::read_cols(gt + 32 * t * TL::PITCH, ca, s), vs, dp);
                    }
                    floatx16 x = value(sc);
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int4 s4 = *reinterpret_cast<const int4 *>(st + at + 8 * i);
                            const int sees4[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (key >= sees4[r])
                                    x[4 * i + r] = -HUGE_VALF;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float4 l4 = *reinterpret_cast<const float4 *>(lt + at + 8 * i);
                        const float l[4] = {l4.x, l4.y, l4.z, l4.w};
                        float4 r4{0.f, 0.f, 0.f, 0.f};
                        if constexpr (M::FINE)
                            r4 = *reinterpret_cast<const float4 *>(lt + 3 * BR + at + 8 * i);
                        const float ll[4] = {r4.x, r4.y, r4.z, r4.w};
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float p = prob<M>(x[4 * i + r], a, l[r], ll[r]);
                            x[4 * i + r] = p;
                            dp[4 * i + r] *= p;
                        }
                    }
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const Frag pf = to_frag<M>(x, s), sf = to_frag<M>(dp, s);
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            dva[d] = mma(TL::read_rows(gt, ra, 32 * t + 16 * s, d), pf, dva[d]);
                            dka[d] = mma(TL::read_rows(qt, ra, 32 * t + 16 * s, d), sf, dka[d]);
                        }
                    }
                }
            }
            if (more)
                store(smem + ((j + 1 - tile0) & 1) * BUF);
            __syncthreads();
        }

        if (pc.parts > 1) {
            const int64_t slot = 2 * static_cast<int64_t>(kvh) * pl.shares + pc.slot;
            float4 *part = pl.part + slot * (2 * DT * 4 * NT) + threadIdx.x;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    part[(d * 4 + i) * NT] = quad(dka[d], i);
                    part[((DT + d) * 4 + i) * NT] = quad(dva[d], i);
                }
        } else if (key < m) {
            E *kp = dk + (pc.k0 + key) * gr.lddk + kvh * a.D;
            E *vp = dv + (pc.k0 + key) * gr.lddv + kvh * a.D;
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                store_col(kp, dka[d], 32 * d + 4 * h, a.D, a.scale);
                store_col(vp, dva[d], 32 * d + 4 * h, a.D, 1.f);
            }
        }
        if (threadIdx.x == 0)
            next = after;
        __syncthreads();
        w = __builtin_amdgcn_readfirstlane(next);
        __syncthreads();
    }
}

// Adds up the pieces of divided tiles: block = (head, divided tile, 32 elements
// of dk or dv), thread = the lane that holds them in attn_dkv_k.
template <typename E, int DC, int NT>
__global__ __launch_bounds__(NT) void attn_dkv_join_k(E *dk, E *dv, AttnArgs a, AttnGrads gr,
                                                       KeyPlan pl)
{
    constexpr int DT = DC / 32;
    const int item = blockIdx.x % pl.shares, kvh = blockIdx.x / pl.shares;
    if (item >= pl.ends[kClasses])
        return;
    const KeyPiece pc = pl.divided[item];
    const int which = blockIdx.y; // dk's tiles of 32 elements, then dv's
    floatx16 sum = floatx16{};
    for (int i = 0; i < pc.parts; ++i) {
        const float4 *p = pl.part +
                          (2 * static_cast<int64_t>(kvh) * pl.shares + pc.slot + i) *
                              (2 * DT * 4 * NT) +
                          which * 4 * NT + threadIdx.x;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            add_quad(sum, c, p[c * NT]);
    }
    const int lane = threadIdx.x & 63;
    const int key = pc.key0 + (threadIdx.x >> 6) * 32 + (lane & 31), c0 = 4 * (lane >> 5);
    if (key >= pc.m)
        return;
    const int64_t at = pc.k0 + key;
    if (which < DT)
        store_col(dk + at * gr.lddk + kvh * a.D, sum, 32 * which + c0, a.D, a.scale);
    else
        store_col(dv + at * gr.lddv + kvh * a.D, sum, 32 * (which - DT) + c0, a.D, 1.f);
}

template <typename E, int DC, int NW>
hipError_t launch_dq(const E *q, const E *k, const E *v, const E *o, const float *lse,
                     const E *dout, E *dq, float *delta, AttnArgs a, const AttnGrads &gr,
                     const KeyPlan &pl, hipStream_t st)
{
    constexpr int BK = NW == 2 || (sizeof(E) == 4 && DC > 32) ? 32 : 64;
    a.slots = attn_slots(a.Tq, a.group.G, 32 * NW, a.S);
    // one block more, the first, divides the keys' work
    HEX_LAUNCH((attn_dq_k<Math<E>, DC, BK, NW>), dim3(attn_blocks(a) + 1), dim3(64 * NW), 0, st, q,
               k, v, o, lse, dout, dq, delta, a, gr, pl);
    return hipGetLastError();
}

template <typename E, int DC, int KT>
hipError_t launch_dkv(const E *q, const E *k, const E *v, const float *lse, const E *dout, E *dk,
                      E *dv, const float *delta, const AttnArgs &a, const AttnGrads &gr,
                      const KeyPlan &pl, hipStream_t st)
{
    HEX_LAUNCH((attn_dkv_k<Math<E>, DC, dkv_rows(sizeof(E) == 4, DC), KT>),
               dim3(static_cast<uint32_t>(pl.blocks)), dim3(2 * KT), 0, st, q, k, v, lse, dout,
               delta, dk, dv, a, gr, pl);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !pl.divides)
        return e;
    HEX_LAUNCH((attn_dkv_join_k<E, DC, 2 * KT>),
               dim3(static_cast<uint32_t>(pl.shares) * a.Hkv, DC / 16), dim3(2 * KT), 0, st, dk, dv,
               a, gr, pl);
    return hipGetLastError();
}

template <typename E, int DC>
hipError_t launch(const E *q, const E *k, const E *v, const E *o, const float *lse, const E *dout,
                  E *dq, E *dk, E *dv, float *delta, const AttnArgs &a, const AttnGrads &gr,
                  const KeyPlan &pl, hipStream_t st)
{
    const auto dq_of = [&](auto f) { return f(q, k, v, o, lse, dout, dq, delta, a, gr, pl, st); };
    hipError_t e;
    if constexpr (sizeof(E) == 2)
        e = attn_short(a) ? dq_of(launch_dq<E, DC, 2>) : dq_of(launch_dq<E, DC, 4>);
    else
        e = dq_of(launch_dq<E, DC, 4>);
    if (e != hipSuccess || a.Tk == 0)
        return e;
    if constexpr (dkv_wide(sizeof(E) == 4, DC))
        if (pl.key_tile == 256)
            return launch_dkv<E, DC, 256>(q, k, v, lse, dout, dk, dv, delta, a, gr, pl, st);
    return launch_dkv<E, DC, 128>(q, k, v, lse, dout, dk, dv, delta, a, gr, pl, st);
}

template <typename E>
hipError_t by_dim(const void *q, const void *k, const void *v, const void *o, const float *lse,
                  const void *dout, void *dq, void *dk, void *dv, float *delta, const AttnArgs &a,
                  const AttnGrads &gr, const KeyPlan &pl, hipStream_t st)
{
    const auto run = [&](auto f) {
        return f(static_cast<const E *>(q), static_cast<const E *>(k), static_cast<const E *>(v),
                 static_cast<const E *>(o), lse, static_cast<const E *>(dout), static_cast<E *>(dq),
                 static_cast<E *>(dk), static_cast<E *>(dv), delta, a, gr, pl, st);
    };
    if (a.D <= 32)
        return run(launch<E, 32>);
    if (a.D <= 64)
        return run(launch<E, 64>);
    if (a.D <= 96)
        return run(launch<E, 96>);
    return run(launch<E, 128>);
}

size_t round16(size_t n) { return (n + 15) & ~static_cast<size_t>(15); }

// the workspace: delta, the plan's parts, partial sums
struct BwdSpace {
    size_t before, next, ends, divided, list, part, bytes;
    int shares, blocks, room, row_tile, key_tile;
    bool divides;
};
BwdSpace bwd_space(int Tq, int Tk, int S, int Hq, int Hkv, int D, Dtype dt)
{
    const int DC = (D + 31) / 32 * 32;
    const bool f32 = dt == F32;
    BwdSpace w;
    w.row_tile = dkv_rows(f32, DC);
    // no more shares of a head than make kLeast units each, no more blocks
    // than pieces
    w.key_tile = dkv_wide(f32, DC) && Tk / dkv_wide_keys(DC) >= S ? 256 : 128;
    const double tiles = Tk / w.key_tile + static_cast<double>(S);
    const double units = tiles * (static_cast<double>(Tq) * (Hq / Hkv) / w.row_tile + 1 + kFixed);
    const int held = dkv_waves(f32, DC) * 128 / w.key_tile * device_cus();
    const int most = (kShares * held + Hkv - 1) / Hkv;
    w.shares = units / kLeast + 1 < most ? static_cast<int>(units / kLeast) + 1 : most;
    // a divided tile has more than a share, so that there are fewer of them
    // than shares, and fewer pieces of them than twice that
    w.room = static_cast<int>(tiles) + 2 * w.shares;
    // no tile is divided where one share is all there is, nor one of so few rows
    const int64_t row_tiles = static_cast<int64_t>(Tq) * (Hq / Hkv) / w.row_tile + 1;
    w.divides = w.shares > 1 && row_tiles + kFixed > kLeast;
    w.blocks = static_cast<double>(w.room) * Hkv < held ? w.room * Hkv : held;
    w.before = round16(static_cast<size_t>(Tq) * Hq * sizeof(float));
    w.next = (w.before + static_cast<size_t>(S) * sizeof(int) + 255) & ~static_cast<size_t>(255);
    w.ends = w.next + 256; // the counter in a cache line of its own
    w.divided = w.ends + 256;
    w.list = w.divided + round16(static_cast<size_t>(w.shares) * sizeof(KeyPiece));
    w.part = w.list + round16(static_cast<size_t>(w.room) * sizeof(KeyPiece));
    const size_t parts = w.divides ? static_cast<size_t>(w.shares) * Hkv * 2 : 0;
    w.bytes = w.part + parts * 2 * w.key_tile * DC * sizeof(float);
    return w;
}

} // namespace
} // namespace attn

hipError_t attn_bwd(const void *q, const void *k, const void *v, const void *o, const float *lse,
                    const void *dout, void *dq, void *dk, void *dv, void *ws, const AttnArgs &a,
                    const AttnGrads &gr, Dtype dt, hipStream_t st)
{
    const attn::BwdSpace w = attn::bwd_space(a.Tq, a.Tk, a.S, a.Hq, a.Hkv, a.D, dt);
    unsigned char *p = static_cast<unsigned char *>(ws);
    KeyPlan pl;
    pl.before = reinterpret_cast<int *>(p + w.before);
    pl.next = reinterpret_cast<int *>(p + w.next);
    pl.ends = reinterpret_cast<int *>(p + w.ends);
    pl.divided = reinterpret_cast<KeyPiece *>(p + w.divided);
    pl.list = reinterpret_cast<KeyPiece *>(p + w.list);
    pl.part = reinterpret_cast<float4 *>(p + w.part);
    pl.shares = w.shares;
    pl.blocks = w.blocks;
    pl.room = w.room;
    pl.row_tile = w.row_tile;
    pl.key_tile = w.key_tile;
    pl.divides = w.divides;
    pl.row_shift = w.row_tile == 64 ? 6 : 5;
    float *delta = static_cast<float *>(ws);
    return dt == F32
               ? attn::by_dim<float>(q, k, v, o, lse, dout, dq, dk, dv, delta, a, gr, pl, st)
               : attn::by_dim<bf16raw>(q, k, v, o, lse, dout, dq, dk, dv, delta, a, gr, pl, st);
}

size_t attn_bwd_workspace(int Tq, int Tk, int S, int Hq, int Hkv, int D, Dtype dt)
{
    return attn::bwd_space(Tq, Tk, S, Hq, Hkv, D, dt).bytes;
}

} // namespace hexk
