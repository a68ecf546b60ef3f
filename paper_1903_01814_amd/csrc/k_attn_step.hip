// k_attn_step.hip -- attention of a few new tokens of every sequence over its
// cached keys: the forward for single tokens.
//
// The definition is that of k_attn_fwd.hip; token t of the n new ones sees the
// keys up to its own, which is the (n - t)-th from the end.  The work is
// reading the cache once: a block takes a run of keys of one (sequence, key
// head) for up to 32 rows (new tokens times the query heads that share the key
// head), so that few sequences still fill the card; each of its four waves
// takes every fourth tile of 32 keys by itself, with its own buffers and no
// barrier, the next tile's loads (32 to 64 KB a block) in flight during the
// products.  Most rows of a product are empty, which costs nothing here: the
// matrix cores are busy 0.04 of the time the loads take.  The waves' maxima,
// sums and outputs are joined in LDS, the runs' by attn_join_k (a launch more,
// 4 us; a last block that joins needs fences across dies, not measured here).
// Bound by memory: three sequences of 9000 to 16432 keys, 16 heads of 128 on 4
// in bfloat16, 16.5 us and 4.6 to join (80 MB, 4.8 TB/s; a large copy reaches
// 4.95); 192 of 32 to 4000, two new tokens each, 8 heads of 64 on 2, 21 and 4.3
// (77 MB, 3.7 TB/s: runs of 1408 keys, 492 of the 1152 blocks have any, and the
// longest sequences end last).
#include "attn.h"
#include "kernels.h"

namespace hexk {
namespace attn {
namespace {

constexpr int kStepWaves = 4;
constexpr int kMaxRuns = 1024; // of a row, to be joined in LDS

template <typename M, int DC, typename E = typename M::E>
__global__ __launch_bounds__(64 * kStepWaves, sizeof(E) * DC > 256 ? 1 : 2) void attn_step_k(
    const E *q, const E *k, const E *v, E *o, float *part, float2 *stat, AttnArgs a, StepPlan pl)
{
    constexpr int DT = DC / 32, DS = DC / 16, BK = 32;
    using TL = Tile<M, DC, BK>;
    using Frag = typename M::Frag;
    constexpr int TB = TL::SIZE;
    static_assert(2 * TB >= 32 * DC * 4, "");
    __shared__ __align__(16) unsigned char smem[kStepWaves][2 * TB];
    __shared__ float stats[2][kStepWaves][32];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int h = lane >> 5, col = lane & 31;
    // Runs outermost: late ones, which only long sequences have, are spread
    // over all dies (blocks go to the 8 dies in turn; with the runs inside, the
    // same few dies got them, 19 to 45 us for one batch)
    uint32_t id = blockIdx.x;
    const int kvh = id % a.Hkv;
    id /= a.Hkv;
    const int seq = id % a.S;
    id /= a.S;
    const int rt = id % pl.row_tiles, split = id / pl.row_tiles;
    const Group g = a.group;
    const int rows = pl.n * g.G;

    int kb, m;
    key_span(a, seq, 0, 0, kb, m);
    const int begin = split * pl.chunk, end = min(m, begin + pl.chunk);
    if (begin >= end && !(split == 0 && pl.splits == 1))
        return; // attn_join_k knows

    const int r = rt * 32 + col;
    const int t = row_token(g, min(r, rows - 1));
    const int64_t row = (static_cast<int64_t>(seq) * pl.n + t) * a.Hq + kvh * g.G +
                        (min(r, rows - 1) - t * g.G);
    Frag qf[DS];
#pragma unroll
    for (int s = 0; s < DS; ++s)
        qf[s] = load_frag<M>(q + row * a.D, 16 * s + 8 * h, a.D);
    const int see = r < rows ? max(0, m - pl.n + t + 1) : 0;

    const E *kp = k + kb * a.ldk + kvh * a.D, *vp = v + kb * a.ldv + kvh * a.D;
    unsigned char *kt = smem[wave], *vt = kt + TB;
    Stage<M, DC, BK, 64> ks, vs;
    const uint32_t ldk = a.ldk * sizeof(E), ldv = a.ldv * sizeof(E);
    auto load = [&](int k0) {
        ks.rows(kp + k0 * a.ldk, ldk, m - k0, a.D);
        vs.rows(vp + k0 * a.ldv, ldv, m - k0, a.D);
    };
    auto store = [&]() {
        ks.put(kt);
        vs.put(vt);
    };

    int ca = TL::cols_at(col, h);
    typename TL::RowsAt ra = TL::rows_at(lane);
    floatx16 acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
        acc[d] = floatx16{};
    float mx = -HUGE_VALF, sum = 0.f;

    int k0 = __builtin_amdgcn_readfirstlane(begin + wave * BK);
    if (k0 < end)
        load(k0);
    for (; k0 < end; k0 += kStepWaves * BK) {
        store();
        in_loop(ca), in_loop(ra.a), in_loop(ra.b);
        // one wave's LDS reads and writes keep their order; this keeps the
        // compiler to it
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        if (k0 + kStepWaves * BK < end)
            load(k0 + kStepWaves * BK);
        typename M::Score sc{};
#pragma unroll
        for (int s = 0; s < DS; ++s)
            add_product(TL::read_cols(kt, ca, s), qf[s], sc);
        floatx16 x = value(sc);
        // keys past the run belong to another block or do not exist
        const int left = min(see, end) - k0 - 4 * h;
        float top = -HUGE_VALF;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (8 * (i >> 2) + (i & 3) >= left)
                x[i] = -HUGE_VALF;
            top = fmaxf(top, x[i]);
        }
        top = both_max(top) * a.c;
        const float to = fmaxf(mx, top);
        const float f = mx == -HUGE_VALF ? 0.f : __builtin_amdgcn_exp2f(mx - to);
        mx = to;
        sum *= f;
        const float ref = mx == -HUGE_VALF ? 0.f : mx;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[i] = prob<M>(x[i], a, ref, 0.f);
            sum += x[i];
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
            acc[d] *= f;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const Frag pf = to_frag<M>(x, s);
#pragma unroll
            for (int d = 0; d < DT; ++d)
                acc[d] = mma(TL::read_rows(vt, ra, 16 * s, d), pf, acc[d]);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }

    sum = both_sum(sum);
    if (h == 0) {
        stats[0][wave][col] = mx;
        stats[1][wave][col] = sum;
    }
    __syncthreads();
    float all = stats[0][0][col];
#pragma unroll
    for (int i = 1; i < kStepWaves; ++i)
        all = fmaxf(all, stats[0][i][col]);
    {
        const float f = mx == -HUGE_VALF ? 0.f : __builtin_amdgcn_exp2f(mx - all);
        // [row][head element], 16-byte chunks permuted by the row
        float4 *out = reinterpret_cast<float4 *>(smem[wave]);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = 8 * d + 2 * i + h;
                out[col * (DC / 4) + (c ^ (col & 7))] =
                    float4{acc[d][4 * i] * f, acc[d][4 * i + 1] * f, acc[d][4 * i + 2] * f,
                           acc[d][4 * i + 3] * f};
            }
    }
    __syncthreads();
    // thread: one row's chunks in turn
    for (int e = threadIdx.x; e < 32 * (DC / 4); e += 64 * kStepWaves) {
        const int rr = e / (DC / 4), c = e % (DC / 4);
        const int r2 = rt * 32 + rr;
        if (r2 >= rows || 4 * c >= a.D)
            continue;
        float top = stats[0][0][rr];
#pragma unroll
        for (int i = 1; i < kStepWaves; ++i)
            top = fmaxf(top, stats[0][i][rr]);
        float l = 0.f;
        float4 s{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kStepWaves; ++i) {
            const float mi = stats[0][i][rr];
            if (mi != -HUGE_VALF)
                l += stats[1][i][rr] * __builtin_amdgcn_exp2f(mi - top);
            const float4 u =
                reinterpret_cast<const float4 *>(smem[i])[rr * (DC / 4) + (c ^ (rr & 7))];
            s.x += u.x, s.y += u.y, s.z += u.z, s.w += u.w;
        }
        const int t2 = row_token(g, r2);
        const int64_t out = (static_cast<int64_t>(seq) * pl.n + t2) * a.Hq + kvh * g.G +
                            (r2 - t2 * g.G);
        if (pl.splits == 1) {
            const float f = l == 0.f ? 0.f : 1.f / l;
            store4(o + out * a.D + 4 * c, s.x * f, s.y * f, s.z * f, s.w * f);
        } else {
            const int64_t at = split * pl.rows + out;
            store4(part + at * a.D + 4 * c, s.x, s.y, s.z, s.w);
            if (c == 0)
                stat[at] = float2{top, l};
        }
    }
}

// Joins the runs of a row: block = row, thread = 4 elements and every ny-th run.
// NT threads: a wave up to 16 runs (192 sequences, two tokens, 8 heads: 4.3 us,
// 7.5 with a block), else a block (3 sequences, 16 heads, 40 runs: 4.6, 6.0 with
// a wave).
template <typename E, int NT>
__global__ __launch_bounds__(NT) void attn_join_k(const float *part, const float2 *stat, E *o,
                                                   AttnArgs a, StepPlan pl)
{
    __shared__ float weight[kMaxRuns];
    constexpr int NW = NT / 64;
    __shared__ float red[2][NW];
    __shared__ __align__(16) float4 sums[NT];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    int kb, m;
    key_span(a, static_cast<int>(row / (static_cast<int64_t>(pl.n) * a.Hq)), 0, 0, kb, m);
    const int runs = (m + pl.chunk - 1) / pl.chunk;
    // the largest maximum, then every run's weight and the sum of the weights
    float top = -HUGE_VALF;
    for (int i = tid; i < runs; i += NT)
        top = fmaxf(top, stat[i * pl.rows + row].x);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
        top = fmaxf(top, __shfl_xor(top, d));
    if ((tid & 63) == 0)
        red[0][tid >> 6] = top;
    __syncthreads();
    top = red[0][0];
#pragma unroll
    for (int i = 1; i < NW; ++i)
        top = fmaxf(top, red[0][i]);
    float l = 0.f;
    for (int i = tid; i < runs; i += NT) {
        const float2 st = stat[i * pl.rows + row];
        // a run of which no key is seen has no maximum
        const float w = st.x == -HUGE_VALF ? 0.f : __builtin_amdgcn_exp2f(st.x - top);
        weight[i] = w;
        l = fmaf(st.y, w, l);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
        l += __shfl_xor(l, d);
    if ((tid & 63) == 0)
        red[1][tid >> 6] = l;
    __syncthreads();
    l = red[1][0];
#pragma unroll
    for (int i = 1; i < NW; ++i)
        l += red[1][i];
    const int per = a.D / 4, ny = NT / per;
    const int c = tid % per, y = tid / per;
    float4 s{0, 0, 0, 0};
    if (y < ny)
#pragma unroll 4
        for (int i = y; i < runs; i += ny) {
            const float4 u =
                *reinterpret_cast<const float4 *>(part + (i * pl.rows + row) * a.D + 4 * c);
            const float w = weight[i];
            s.x = fmaf(u.x, w, s.x), s.y = fmaf(u.y, w, s.y);
            s.z = fmaf(u.z, w, s.z), s.w = fmaf(u.w, w, s.w);
        }
    sums[tid] = s;
    __syncthreads();
    if (y != 0)
        return;
    for (int i = 1; i < ny; ++i) {
        const float4 u = sums[i * per + c];
        s.x += u.x, s.y += u.y, s.z += u.z, s.w += u.w;
    }
    const float f = l == 0.f ? 0.f : 1.f / l;
    store4(o + row * a.D + 4 * c, s.x * f, s.y * f, s.z * f, s.w * f);
}

template <typename E, int DC>
hipError_t launch(const void *q, const void *k, const void *v, void *o, void *ws,
                  const AttnArgs &a, const StepPlan &pl, hipStream_t st)
{
    float *part = static_cast<float *>(ws);
    float2 *stat =
        reinterpret_cast<float2 *>(part + static_cast<int64_t>(pl.splits) * pl.rows * a.D);
    const uint32_t blocks = static_cast<uint32_t>(a.S) * pl.row_tiles * pl.splits * a.Hkv;
    using M = std::conditional_t<sizeof(E) == 2, Bf16, Full>;
    HEX_LAUNCH((attn_step_k<M, DC>), dim3(blocks), dim3(64 * kStepWaves), 0, st,
               static_cast<const E *>(q), static_cast<const E *>(k), static_cast<const E *>(v),
               static_cast<E *>(o), part, stat, a, pl);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || pl.splits == 1)
        return e;
    if (pl.splits <= 16)
        HEX_LAUNCH((attn_join_k<E, 64>), dim3(static_cast<uint32_t>(pl.rows)), dim3(64), 0, st,
                   part, stat, static_cast<E *>(o), a, pl);
    else
        HEX_LAUNCH((attn_join_k<E, 256>), dim3(static_cast<uint32_t>(pl.rows)), dim3(256), 0, st,
                   part, stat, static_cast<E *>(o), a, pl);
    return hipGetLastError();
}

template <typename E>
hipError_t by_dim(const void *q, const void *k, const void *v, void *o, void *ws,
                  const AttnArgs &a, const StepPlan &pl, hipStream_t st)
{
    if (a.D <= 32)
        return launch<E, 32>(q, k, v, o, ws, a, pl, st);
    if (a.D <= 64)
        return launch<E, 64>(q, k, v, o, ws, a, pl, st);
    if (a.D <= 96)
        return launch<E, 96>(q, k, v, o, ws, a, pl, st);
    return launch<E, 128>(q, k, v, o, ws, a, pl, st);
}

} // namespace
} // namespace attn

StepPlan step_plan(int S, int n, int Hq, int Hkv, int max_len)
{
    StepPlan p;
    p.n = n;
    p.rows = static_cast<int64_t>(S) * n * Hq;
    p.row_tiles = (n * (Hq / Hkv) + 31) / 32;
    const int64_t one = static_cast<int64_t>(S) * Hkv * p.row_tiles;
    // Few sequences: as many blocks as the card holds (16 heads of 128 on 4,
    // three of 9000 to 16432 keys: 22.5 us with two a unit, 25.3 with four).
    // Many: their lengths differ, and finer runs even them out (192 of 32 to
    // 4000 keys, 8 heads of 64 on 2: 26.7 us with four, 29.7 with two).
    const int per_cu = one * 8 <= device_cus() ? 2 : 4;
    constexpr int step = 32 * attn::kStepWaves; // keys a block takes in one turn
    const int64_t most = (static_cast<int64_t>(max_len) + step - 1) / step;
    const int64_t want = (per_cu * static_cast<int64_t>(device_cus()) + one - 1) / one;
    int64_t splits = want < 1 || most < 1 ? 1 : want < most ? want : most;
    if (splits > attn::kMaxRuns)
        splits = attn::kMaxRuns;
    p.chunk = static_cast<int>((most + splits - 1) / splits) * step;
    if (p.chunk < step)
        p.chunk = step;
    const int64_t len = max_len;
    p.splits = most < 1 ? 1 : static_cast<int>((len + p.chunk - 1) / p.chunk);
    return p;
}

size_t step_workspace(const StepPlan &p, int D)
{
    return p.splits == 1 ? 0 : static_cast<size_t>(p.splits) * p.rows * (D + 2) * sizeof(float);
}

hipError_t attn_step(const void *q, const void *k, const void *v, void *o, void *ws,
                     const AttnArgs &a, const StepPlan &pl, Dtype dt, hipStream_t st)
{
    return dt == F32 ? attn::by_dim<float>(q, k, v, o, ws, a, pl, st)
                     : attn::by_dim<bf16raw>(q, k, v, o, ws, a, pl, st);
}

} // namespace hexk
