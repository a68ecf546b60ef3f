// k_attn_fwd.hip -- softmax attention over packed sequences, forward.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(x_ij - lse_i),  x_ij = scale q_i . k_j,
//   lse_i = log sum_j exp(x_ij)
//
// in one pass over the keys with a running maximum m and sum l per row.  A
// block owns TR = 128 NQ rows of one key head of one sequence (a row is a
// query token and one of the G query heads that share the key head, so short
// sequences fill a tile G times better and the keys are read once for the
// group), a wave 32 NQ of them.  Per tile of BK keys, staged in LDS for the
// whole block (two buffers, the next tile's loads in flight during the
// products):
//   X^T = K Q^T   keys as rows: a lane holds one query's scores
//   p = 2^(x c - m)  with c = scale log2(e), m and l in the lane
//   O^T += V^T P^T   P^T straight from the registers, V^T by the transposing read
// The maximum is raised only when a row passes it by more than 2^kSlack: the
// sums stay exact in float32, and most tiles save the rescaling of O.
#include "attn.h"
#include "kernels.h"

namespace hexk {
namespace attn {
namespace {

constexpr float kSlack = 8.f; // in powers of two

// NQ blocks of 32 rows a wave, BK keys a tile.
template <typename E, int DC, int NQ, int BK>
__global__ __launch_bounds__(256, 2) void attn_fwd_k(const E *q, const E *k, const E *v, E *o,
                                                  float *lse, AttnArgs a)
{
    using TL = Tile<E, DC>;
    using Frag = typename Elem<E>::Frag;
    constexpr int TR = 128 * NQ, KT = BK / 32, DT = DC / 32, DS = DC / 16;
    constexpr int TB = TL::bytes(BK);
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

    // this lane's query of each block of rows, and how many keys it sees
    Frag qf[NQ][DS];
    int see[NQ], most = 0;
    int64_t at[NQ];
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
        const int r = row0 + (wave * NQ + b) * 32 + col;
        const int rc = min(r, rows - 1);
        const int t = row_token(g, rc);
        const int head = kvh * g.G + rc - t * g.G;
        at[b] = static_cast<int64_t>(sp.begin + t) * a.Hq + head;
        const E *qp = q + (sp.begin + t) * a.ldq + head * a.D;
#pragma unroll
        for (int s = 0; s < DS; ++s)
            qf[b][s] = load_frag<E>(qp, 16 * s + 8 * h, a.D);
        see[b] = r < rows ? (a.causal ? min(m, max(0, t + ahead + 1)) : m) : 0;
        most = max(most, see[b]);
    }
    // keys that any row of the wave, and of the block, sees; and that all do
    const int r_last = min(rows, row0 + TR) - 1;
    const int end = a.causal ? min(m, max(0, row_token(g, r_last) + ahead + 1)) : m;
    const int ntiles = (end + BK - 1) / BK;
    int least = see[0];
#pragma unroll
    for (int b = 1; b < NQ; ++b)
        least = min(least, see[b]);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        most = max(most, __shfl_xor(most, d));
        least = min(least, __shfl_xor(least, d));
    }
    most = __builtin_amdgcn_readfirstlane(most);
    least = __builtin_amdgcn_readfirstlane(least);

    const E *kp = k + kb * a.ldk + kvh * a.D, *vp = v + kb * a.ldv + kvh * a.D;
    Stage<E, DC, BK, 256> ks, vs;
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
    floatx16 acc[NQ][DT];
    float mx[NQ], sum[NQ];
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
        mx[b] = -HUGE_VALF;
        sum[b] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
            acc[b][d] = floatx16{};
    }

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
            floatx16 x[NQ][KT];
#pragma unroll
            for (int t = 0; t < KT; ++t) {
#pragma unroll
                for (int b = 0; b < NQ; ++b)
                    x[b][t] = floatx16{};
#pragma unroll
                for (int s = 0; s < DS; ++s) {
                    const Frag kf = TL::read_cols(kt + 32 * t * TL::PITCH, ca, s);
#pragma unroll
                    for (int b = 0; b < NQ; ++b)
                        x[b][t] = add_product(kf, qf[b][s], x[b][t]);
                }
            }
            if ((j + 1) * BK > least) {
#pragma unroll
                for (int b = 0; b < NQ; ++b) {
                    const int left = see[b] - j * BK - 4 * h;
#pragma unroll
                    for (int t = 0; t < KT; ++t)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (32 * t + 8 * (r >> 2) + (r & 3) >= left)
                                x[b][t][r] = -HUGE_VALF;
                }
            }
#pragma unroll
            for (int b = 0; b < NQ; ++b) {
                float top = x[b][0][0];
#pragma unroll
                for (int t = 0; t < KT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        top = fmaxf(top, x[b][t][r]);
                top = both_max(top) * a.c;
                if (__any(top > mx[b] + kSlack)) {
                    const float to = fmaxf(mx[b], top);
                    const float f = mx[b] == -HUGE_VALF ? 0.f : __builtin_amdgcn_exp2f(mx[b] - to);
                    mx[b] = to;
                    sum[b] *= f;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
                        acc[b][d] *= f;
                }
                // a row that has seen no key: every p is 0
                const float ref = mx[b] == -HUGE_VALF ? 0.f : mx[b];
#pragma unroll
                for (int t = 0; t < KT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float p = prob<E>(x[b][t][r], a, ref, 0.f);
                        x[b][t][r] = p;
                        sum[b] += p;
                    }
            }
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    Frag pf[NQ];
#pragma unroll
                    for (int b = 0; b < NQ; ++b)
                        pf[b] = to_frag<E>(x[b][t], s);
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const Frag vf = TL::read_rows(vt, ra, 32 * t + 16 * s, d);
#pragma unroll
                        for (int b = 0; b < NQ; ++b)
                            acc[b][d] = mma(vf, pf[b], acc[b][d]);
                    }
                }
        }
        if (more)
            store(smem + ((j + 1) & 1) * 2 * TB);
        __syncthreads();
    }

#pragma unroll
    for (int b = 0; b < NQ; ++b) {
        const float l = both_sum(sum[b]);
        const int r = row0 + (wave * NQ + b) * 32 + col;
        if (r >= rows)
            continue;
        const float f = l == 0.f ? 0.f : 1.f / l;
        // at = token * Hq + head
        const int64_t token = at[b] / a.Hq;
        E *op = o + token * a.ldo + (at[b] - token * a.Hq) * a.D;
#pragma unroll
        for (int d = 0; d < DT; ++d)
            store_col(op, acc[b][d], 32 * d + 4 * h, a.D, f);
        if (lse != nullptr && h == 0)
            lse[at[b]] = l == 0.f ? -HUGE_VALF : log_sum(mx[b], l);
    }
}

template <typename E, int DC>
hipError_t launch(const void *q, const void *k, const void *v, void *o, float *lse, AttnArgs a,
                  hipStream_t st)
{
    constexpr bool F32 = sizeof(E) == 4;
    constexpr int NQ = 1, BK = F32 && DC > 64 ? 32 : 64;
    a.slots = attn_slots(a.Tq, a.group.G, 128 * NQ, a.S);
    HEX_LAUNCH((attn_fwd_k<E, DC, NQ, BK>), dim3(attn_blocks(a)), dim3(256),
               0, st, static_cast<const E *>(q), static_cast<const E *>(k),
               static_cast<const E *>(v), static_cast<E *>(o), lse, a);
    return hipGetLastError();
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
