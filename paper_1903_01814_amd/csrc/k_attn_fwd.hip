// k_attn_fwd.hip -- softmax attention over packed sequences, forward.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(x_ij - lse_i),  x_ij = scale q_i . k_j,
//   lse_i = log sum_j exp(x_ij)
//
// in one pass over the keys with a running maximum m and sum l per row.  A
// block owns 128 rows (64 where sequences are short) of one key head of one
// sequence (a row is a query token and one of the G query heads that share the
// key head, so short sequences fill a tile G times better and the keys are
// read once for the group), a wave 32 of them.  Per tile of BK keys, staged in
// LDS for the whole block (two buffers, the next tile's loads in flight during
// the products):
//   X^T = K Q^T   keys as rows: a lane holds one query's scores
//   p = 2^(x c - m)  with c = scale log2(e), m and l in the lane
//   O^T += V^T P^T   P^T straight from the registers, V^T by the transposing read
// The maximum is raised only when a row passes it by more than 2^kSlack: the
// sums stay exact in float32, and most tiles save the rescaling of O.
//
// Bound by the matrix cores and the vector unit in turn: one wave's exponentials
// (a quarter of the rate) run beside the other's products, so the two waves a
// SIMD that the launch bounds ask for are worth more than registers (one wave
// with twice as many took 1826 us where two took 1182).  Heads of 128 in
// bfloat16, 16 on 4: one sequence of 16432, causal, 1150 to 1190 us, 930 to 960
// TFLOP/s (a large library product 1220), matrix cores busy 0.47 of the cycles,
// vector unit 0.52; 24 of 500 to 5000, causal 700 us, 780 TFLOP/s.  Heads of 64
// in float32, 16 of 1027: 231 us, 150 TFLOP/s.  Many short sequences of narrow
// heads are bound by memory, by keys that several dies fetch (head_and_slot):
// heads of 32, 512 sequences of 20 to 400, 62 us for 296 MB read and 39 written,
// 5.4 TB/s, where 135 MB in all would do.
#include "attn.h"
#include "kernels.h"

namespace hexk {
namespace attn {
namespace {

constexpr float kSlack = 8.f; // in powers of two

// NW waves, BK keys a tile: 64 for heads up to 64 (in bfloat16; 24 sequences of
// 500 to 5000: 362 us, with 32 keys 391) and up to 32 in float32, else 32: three
// waves a SIMD fit then instead of two (heads of 128: 24 of 2048 keys 963 ->
// 919 us, 64 of 470 146 -> 135, 128 of 370 263 -> 244, one of 16432 1125 ->
// 1150, two of them the same).
template <typename M, int DC, int BK, int NW, typename E = typename M::E>
__global__ __launch_bounds__(64 * NW, attn_waves(sizeof(E) == 4, DC)) void
attn_fwd_k(const E *q, const E *k, const E *v, E *o, float *lse, AttnArgs a)
{
    using TL = Tile<M, DC, BK>;
    using Frag = typename M::Frag;
    constexpr int TR = 32 * NW, KT = BK / 32, DT = DC / 32, DS = DC / 16;
    constexpr int TB = TL::SIZE;
    __shared__ __align__(16) unsigned char smem[4 * TB]; // K, V, K, V

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int h = lane >> 5, col = lane & 31;
    int kvh, w;
    head_and_slot(a, blockIdx.x, kvh, w);
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
    const int ahead = m - sp.n; // causal: query i sees keys up to i + ahead

    // this lane's query, and how many keys it sees
    const int row = row0 + wave * 32 + col, rc = min(row, rows - 1);
    const int tq = row_token(g, rc), head = kvh * g.G + rc - tq * g.G;
    const int64_t token = sp.begin + tq;
    const int see = row < rows ? (a.causal ? min(m, max(0, tq + ahead + 1)) : m) : 0;
    const E *qp = q + token * a.ldq + head * a.D;
    Frag qf[DS];
#pragma unroll
    for (int s = 0; s < DS; ++s)
        qf[s] = load_frag<M>(qp, 16 * s + 8 * h, a.D);
    // keys that any row of the block sees; of the wave; and that all of it see
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
    float mx = -HUGE_VALF, sum = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
        acc[d] = floatx16{};

    // the tile of keys at kt and vt, key0 the first
    auto tile = [&](unsigned char *kt, unsigned char *vt, int key0) {
        // scores before the other waves' vector work (16 heads of 128 on 4: 24
        // sequences of 2048 932 -> 918 us; the exponentials first lost 3 %)
        __builtin_amdgcn_s_setprio(1);
        floatx16 x[KT];
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            typename M::Score sc{};
#pragma unroll
            for (int s = 0; s < DS; ++s)
                add_product(TL::read_cols(kt + 32 * t * TL::PITCH, ca, s), qf[s], sc);
            x[t] = value(sc);
        }
        __builtin_amdgcn_s_setprio(0);
        if (key0 + BK > least) {
            const int left = see - key0 - 4 * h;
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (32 * t + 8 * (r >> 2) + (r & 3) >= left)
                        x[t][r] = -HUGE_VALF;
        }
        float top = x[0][0];
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                top = fmaxf(top, x[t][r]);
        top = both_max(top) * a.c;
        if (__any(top > mx + kSlack)) {
            const float to = fmaxf(mx, top);
            const float f = mx == -HUGE_VALF ? 0.f : __builtin_amdgcn_exp2f(mx - to);
            mx = to;
            sum *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d)
                acc[d] *= f;
        }
        // a row that has seen no key: every p is 0
        const float ref = mx == -HUGE_VALF ? 0.f : mx;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = prob<M>(x[t][r], a, ref, 0.f);
                x[t][r] = p;
                sum += p;
            }
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const Frag pf = to_frag<M>(x[t], s);
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    acc[d] = mma(TL::read_rows(vt, ra, 32 * t + 16 * s, d), pf, acc[d]);
            }
    };

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
        if (j * BK < most)
            tile(kt, vt, j * BK);
        if (more)
            store(smem + ((j + 1) & 1) * 2 * TB);
        __syncthreads();
    }

    const float l = both_sum(sum);
    if (row >= rows)
        return;
    const float f = l == 0.f ? 0.f : __builtin_amdgcn_rcpf(l);
    E *op = o + token * a.ldo + head * a.D;
#pragma unroll
    for (int d = 0; d < DT; ++d)
        store_col(op, acc[d], 32 * d + 4 * h, a.D, f);
    if (lse != nullptr && h == 0)
        lse[token * a.Hq + head] = l == 0.f ? -HUGE_VALF : log_sum(mx, l);
}

template <typename E, int DC, int NW>
hipError_t launch_waves(const E *q, const E *k, const E *v, E *o, float *lse, AttnArgs a,
                        hipStream_t st)
{
    constexpr int BK = NW == 2 || DC > (sizeof(E) == 4 ? 32 : 64) ? 32 : 64;
    a.slots = attn_slots(a.Tq, a.group.G, 32 * NW, a.S);
    HEX_LAUNCH((attn_fwd_k<Math<E>, DC, BK, NW>), dim3(attn_blocks(a)), dim3(64 * NW), 0, st, q, k,
               v, o, lse, a);
    return hipGetLastError();
}

template <typename E, int DC>
hipError_t launch(const void *q, const void *k, const void *v, void *o, float *lse,
                  const AttnArgs &a, hipStream_t st)
{
    const auto run = [&](auto f) {
        return f(static_cast<const E *>(q), static_cast<const E *>(k), static_cast<const E *>(v),
                 static_cast<E *>(o), lse, a, st);
    };
    if constexpr (sizeof(E) == 2)
        if (attn_short(a))
            return run(launch_waves<E, DC, 2>);
    return run(launch_waves<E, DC, 4>);
}

template <typename E>
hipError_t by_dim(const void *q, const void *k, const void *v, void *o, float *lse,
                  const AttnArgs &a, hipStream_t st)
{
    if (a.D <= 32)
        return launch<E, 32>(q, k, v, o, lse, a, st);
    if (a.D <= 64)
        return launch<E, 64>(q, k, v, o, lse, a, st);
    if (a.D <= 96)
        return launch<E, 96>(q, k, v, o, lse, a, st);
    return launch<E, 128>(q, k, v, o, lse, a, st);
}

} // namespace
} // namespace attn

hipError_t attn_fwd(const void *q, const void *k, const void *v, void *o, float *lse,
                    const AttnArgs &a, Dtype dt, hipStream_t st)
{
    return dt == F32 ? attn::by_dim<float>(q, k, v, o, lse, a, st)
                     : attn::by_dim<bf16raw>(q, k, v, o, lse, a, st);
}

} // namespace hexk
