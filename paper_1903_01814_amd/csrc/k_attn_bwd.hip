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
// and do . v are computed twice, 7 products in place of 5; in exchange
// nothing is added through memory, every sum has one order and the result is
// the same from run to run.
#include "attn.h"
#include "kernels.h"

namespace hexk {
namespace attn {
namespace {

// ---- dq: rows as in the forward, 32 NQ a wave, BK keys a tile.
//   X^T = K Q^T and dP^T = V dO^T (keys as rows), dQ^T += K^T dS^T
template <typename E, int DC, int NQ, int BK>
__global__ __launch_bounds__(256, 2) void attn_dq_k(const E *q, const E *k, const E *v, const E *o,
                                                 const float *lse, const E *dout, E *dq,
                                                 float *delta, AttnArgs a, AttnGrads gr)
{
    using TL = Tile<E, DC>;
    using Frag = typename Elem<E>::Frag;
    constexpr int TR = 128 * NQ, KT = BK / 32, DT = DC / 32, DS = DC / 16;
    constexpr int TB = TL::bytes(BK);
    constexpr int NCH = BK * TL::CPR / 256;
    static_assert(BK * TL::CPR % 256 == 0, "");
    __shared__ __align__(16) unsigned char smem[4 * TB]; // K, V, K, V

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int h = lane >> 5, col = lane & 31;
    const int kvh = blockIdx.x % a.Hkv;
    const int w = a.slots - 1 - static_cast<int>(blockIdx.x / a.Hkv);
    const Group g = a.group;
    const Span sp = find_span<TR>(a.q_start, a.S, a.Tq, g.G, w);
    const int rows = sp.n * g.G;
    if (static_cast<int64_t>(sp.tile) * TR >= rows)
        return;
    const int row0 = sp.tile * TR;
    int kb, m;
    key_span(a, sp.seq, kb, m);
    const int ahead = m - sp.n;

    Frag qf[NQ][DS], gf[NQ][DS];
    int see[NQ], most = 0;
    int64_t token[NQ];
    int head[NQ];
    Ref ref[NQ];
    float dl[NQ];
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
        const int r = row0 + (wave * NQ + b) * 32 + col;
        const int rc = min(r, rows - 1);
        const int t = row_token(g, rc);
        head[b] = kvh * g.G + rc - t * g.G;
        token[b] = sp.begin + t;
        const E *qp = q + token[b] * a.ldq + head[b] * a.D;
        const E *gp = dout + token[b] * gr.lddo + head[b] * a.D;
        const E *op = o + token[b] * a.ldo + head[b] * a.D;
        float sum = 0.f;
#pragma unroll
        for (int s = 0; s < DS; ++s) {
            qf[b][s] = load_frag<E>(qp, 16 * s + 8 * h, a.D);
            gf[b][s] = load_frag<E>(gp, 16 * s + 8 * h, a.D);
            const Frag of = load_frag<E>(op, 16 * s + 8 * h, a.D);
            sum += dot8(gf[b][s], of);
        }
        dl[b] = both_sum(sum);
        const float l = lse[token[b] * a.Hq + head[b]];
        // a row that saw no key: every p is 0
        ref[b] = l == -HUGE_VALF ? Ref{HUGE_VALF, 0.f} : ref_of_lse(l);
        if (r < rows && h == 0)
            delta[token[b] * a.Hq + head[b]] = dl[b];
        see[b] = r < rows ? (a.causal ? min(m, max(0, t + ahead + 1)) : m) : 0;
        most = max(most, see[b]);
    }
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
    uint4 ks[NCH], vs[NCH];
    auto load = [&](int tile) {
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int e = threadIdx.x + 256 * i;
            const int c = e % TL::CPR * Elem<E>::VEC;
            const int64_t r = min(tile * BK + e / TL::CPR, m - 1);
            ks[i] = vs[i] = uint4{0, 0, 0, 0};
            if (c < a.D) {
                ks[i] = *reinterpret_cast<const uint4 *>(kp + r * a.ldk + c);
                vs[i] = *reinterpret_cast<const uint4 *>(vp + r * a.ldv + c);
            }
        }
    };
    auto store = [&](unsigned char *t) {
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int e = threadIdx.x + 256 * i;
            const int p = TL::chunk_at(e / TL::CPR, e % TL::CPR);
            *reinterpret_cast<uint4 *>(t + p) = ks[i];
            *reinterpret_cast<uint4 *>(t + TB + p) = vs[i];
        }
    };

    floatx16 acc[NQ][DT];
#pragma unroll
    for (int b = 0; b < NQ; ++b)
#pragma unroll
        for (int d = 0; d < DT; ++d)
            acc[b][d] = floatx16{};

    if (ntiles > 0) {
        load(0);
        store(smem);
    }
    __syncthreads();
    for (int j = 0; j < ntiles; ++j) {
        unsigned char *kt = smem + (j & 1) * 2 * TB, *vt = kt + TB;
        const bool more = j + 1 < ntiles;
        if (more)
            load(j + 1);
        if (j * BK < most) {
            const bool masked = (j + 1) * BK > least;
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                floatx16 x[NQ], dp[NQ];
#pragma unroll
                for (int b = 0; b < NQ; ++b)
                    x[b] = dp[b] = floatx16{};
#pragma unroll
                for (int s = 0; s < DS; ++s) {
                    const Frag kf = TL::read_cols(kt, 32 * t + col, s, h);
                    const Frag vf = TL::read_cols(vt, 32 * t + col, s, h);
#pragma unroll
                    for (int b = 0; b < NQ; ++b) {
                        x[b] = add_product(kf, qf[b][s], x[b]);
                        dp[b] = add_product(vf, gf[b][s], dp[b]);
                    }
                }
#pragma unroll
                for (int b = 0; b < NQ; ++b) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float p = prob<E>(x[b][r], a, ref[b].hi, ref[b].lo);
                        x[b][r] = p * (dp[b][r] - dl[b]);
                    }
                    if (masked) {
                        const int left = see[b] - j * BK - 4 * h;
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (32 * t + 8 * (r >> 2) + (r & 3) >= left)
                                x[b][r] = 0.f;
                    }
                }
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    Frag sf[NQ];
#pragma unroll
                    for (int b = 0; b < NQ; ++b)
                        sf[b] = to_frag<E>(x[b], s);
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const Frag kf = TL::read_rows(kt, 32 * t + 16 * s, d, lane);
#pragma unroll
                        for (int b = 0; b < NQ; ++b)
                            acc[b][d] = mma(kf, sf[b], acc[b][d]);
                    }
                }
            }
        }
        if (more)
            store(smem + ((j + 1) & 1) * 2 * TB);
        __syncthreads();
    }

#pragma unroll
    for (int b = 0; b < NQ; ++b) {
        if (row0 + (wave * NQ + b) * 32 + col >= rows)
            continue;
        E *p = dq + token[b] * gr.lddq + head[b] * a.D;
#pragma unroll
        for (int d = 0; d < DT; ++d)
            store_col(p, acc[b][d], 32 * d + 4 * h, a.D, a.scale);
    }
}

// ---- dk and dv: 128 keys a block, 32 a wave; BR rows a tile.
//   X = Q K^T and dP = dO V^T (query rows as rows; a lane holds one key),
//   dV^T += dO^T P, dK^T += Q^T dS
template <typename E, int DC, int BR>
__global__ __launch_bounds__(256, 2) void attn_dkv_k(const E *q, const E *k, const E *v,
                                                  const float *lse, const E *dout,
                                                  const float *delta, E *dk, E *dv, AttnArgs a,
                                                  AttnGrads gr)
{
    using TL = Tile<E, DC>;
    using Frag = typename Elem<E>::Frag;
    constexpr int RT = BR / 32, DT = DC / 32, DS = DC / 16;
    constexpr int TB = TL::bytes(BR);
    constexpr int NCH = BR * TL::CPR / 256;
    static_assert(BR * TL::CPR % 256 == 0 && BR <= 64, "");
    constexpr int BUF = 2 * TB + 4 * BR * 4; // Q, dO; lse, delta, keys seen, lse's rest
    // the values' operands stay in registers where they fit beside the sums
    constexpr bool VL = DT > 2;
    __shared__ __align__(16) unsigned char smem[2 * BUF + (VL ? TL::bytes(128) : 0)];
    unsigned char *vl = smem + 2 * BUF;

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int h = lane >> 5, col = lane & 31;
    const int kvh = blockIdx.x % a.Hkv;
    const Group g = a.group;
    const Span sp =
        find_span<128>(a.k_start, a.S, a.Tk, 1, static_cast<int>(blockIdx.x / a.Hkv));
    const int m = sp.n;
    if (static_cast<int64_t>(sp.tile) * 128 >= m)
        return;
    const int key0 = sp.tile * 128;
    const int qb = clamp_start(a.q_start, sp.seq, a.Tq);
    const int n = max(0, clamp_start(a.q_start, sp.seq + 1, a.Tq) - qb);
    const int rows = n * g.G, ahead = m - n;

    const int key = key0 + wave * 32 + col, kc = min(key, m - 1);
    Frag kf[DS], vf[VL ? 1 : DS];
#pragma unroll
    for (int s = 0; s < DS; ++s) {
        kf[s] = load_frag<E>(k + (sp.begin + kc) * a.ldk + kvh * a.D, 16 * s + 8 * h, a.D);
        if constexpr (!VL)
            vf[s] = load_frag<E>(v + (sp.begin + kc) * a.ldv + kvh * a.D, 16 * s + 8 * h, a.D);
    }
    if constexpr (VL)
        for (int e = threadIdx.x; e < 128 * TL::CPR; e += 256) {
            const int c = e % TL::CPR * Elem<E>::VEC;
            const int64_t r = sp.begin + min(key0 + e / TL::CPR, m - 1);
            *reinterpret_cast<uint4 *>(vl + TL::chunk_at(e / TL::CPR, e % TL::CPR)) =
                c < a.D ? *reinterpret_cast<const uint4 *>(v + r * a.ldv + kvh * a.D + c)
                        : uint4{0, 0, 0, 0};
        }
    // first row that sees a key of the block
    const int tile0 = a.causal ? static_cast<int>(static_cast<int64_t>(max(0, key0 - ahead)) * g.G / BR) : 0;
    const int ntiles = (rows + BR - 1) / BR;

    const E *qp = q + qb * a.ldq + static_cast<int64_t>(kvh) * g.G * a.D;
    const E *gp = dout + qb * gr.lddo + static_cast<int64_t>(kvh) * g.G * a.D;
    const float *lp = lse + static_cast<int64_t>(qb) * a.Hq + kvh * g.G;
    const float *dp0 = delta + static_cast<int64_t>(qb) * a.Hq + kvh * g.G;
    uint4 qs[NCH], gs[NCH];
    Ref ls{0.f, 0.f};
    float ds = 0.f;
    int sees = 0;
    auto load = [&](int tile) {
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int e = threadIdx.x + 256 * i;
            const int c = e % TL::CPR * Elem<E>::VEC;
            const int r = min(tile * BR + e / TL::CPR, rows - 1);
            const int t = row_token(g, r), hd = r - t * g.G;
            qs[i] = gs[i] = uint4{0, 0, 0, 0};
            if (c < a.D) {
                qs[i] = *reinterpret_cast<const uint4 *>(qp + t * a.ldq + hd * a.D + c);
                gs[i] = *reinterpret_cast<const uint4 *>(gp + t * gr.lddo + hd * a.D + c);
            }
        }
        if (threadIdx.x < BR) {
            const int r = tile * BR + threadIdx.x;
            const int t = row_token(g, min(r, rows - 1)), hd = min(r, rows - 1) - t * g.G;
            const float l = lp[static_cast<int64_t>(t) * a.Hq + hd];
            // rows past the end and rows that saw no key: every p is 0
            ls = r >= rows || l == -HUGE_VALF ? Ref{HUGE_VALF, 0.f} : ref_of_lse(l);
            ds = dp0[static_cast<int64_t>(t) * a.Hq + hd];
            sees = r >= rows ? 0 : a.causal ? max(0, t + ahead + 1) : m;
        }
    };
    auto store = [&](unsigned char *t) {
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int e = threadIdx.x + 256 * i;
            const int p = TL::chunk_at(e / TL::CPR, e % TL::CPR);
            *reinterpret_cast<uint4 *>(t + p) = qs[i];
            *reinterpret_cast<uint4 *>(t + TB + p) = gs[i];
        }
        if (threadIdx.x < BR) {
            float *f = reinterpret_cast<float *>(t + 2 * TB);
            f[threadIdx.x] = ls.hi;
            f[BR + threadIdx.x] = ds;
            reinterpret_cast<int *>(f)[2 * BR + threadIdx.x] = sees;
            f[3 * BR + threadIdx.x] = ls.lo;
        }
    };

    floatx16 dka[DT], dva[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
        dka[d] = dva[d] = floatx16{};

    if (tile0 < ntiles) {
        load(tile0);
        store(smem);
    }
    __syncthreads();
    for (int j = tile0; j < ntiles; ++j) {
        unsigned char *qt = smem + ((j - tile0) & 1) * BUF, *gt = qt + TB;
        const float *lt = reinterpret_cast<const float *>(qt + 2 * TB), *dt = lt + BR;
        const int *st = reinterpret_cast<const int *>(dt + BR);
        const bool more = j + 1 < ntiles;
        if (more)
            load(j + 1);
        // the first row of a tile sees the fewest keys, the last (of the rows
        // there are) the most
        const int first_sees = a.causal ? row_token(g, min(j * BR, rows - 1)) + ahead + 1 : m;
        const int last_sees =
            a.causal ? row_token(g, min((j + 1) * BR, rows) - 1) + ahead + 1 : m;
        const int wkey = key0 + wave * 32;
        if (wkey < last_sees) {
            const bool masked = wkey + 32 > first_sees;
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                floatx16 x = floatx16{}, dp = floatx16{};
#pragma unroll
                for (int s = 0; s < DS; ++s) {
                    x = add_product(TL::read_cols(qt, 32 * t + col, s, h), kf[s], x);
                    const Frag vs = VL ? TL::read_cols(vl, wave * 32 + col, s, h) : vf[VL ? 0 : s];
                    dp = add_product(TL::read_cols(gt, 32 * t + col, s, h), vs, dp);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = 32 * t + 8 * i + 4 * h;
                    const float4 l4 = *reinterpret_cast<const float4 *>(lt + at);
                    const float4 d4 = *reinterpret_cast<const float4 *>(dt + at);
                    const float l[4] = {l4.x, l4.y, l4.z, l4.w}, dd[4] = {d4.x, d4.y, d4.z, d4.w};
                    float4 r4{0.f, 0.f, 0.f, 0.f};
                    if constexpr (sizeof(E) == 4)
                        r4 = *reinterpret_cast<const float4 *>(lt + 3 * BR + at);
                    const float ll[4] = {r4.x, r4.y, r4.z, r4.w};
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float p = prob<E>(x[4 * i + r], a, l[r], ll[r]);
                        x[4 * i + r] = p;
                        dp[4 * i + r] = p * (dp[4 * i + r] - dd[r]);
                    }
                    if (masked) {
                        const int4 s4 = *reinterpret_cast<const int4 *>(st + at);
                        const int sees4[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (key >= sees4[r])
                                x[4 * i + r] = dp[4 * i + r] = 0.f;
                    }
                }
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const Frag pf = to_frag<E>(x, s), sf = to_frag<E>(dp, s);
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        dva[d] = mma(TL::read_rows(gt, 32 * t + 16 * s, d, lane), pf, dva[d]);
                        dka[d] = mma(TL::read_rows(qt, 32 * t + 16 * s, d, lane), sf, dka[d]);
                    }
                }
            }
        }
        if (more)
            store(smem + ((j + 1 - tile0) & 1) * BUF);
        __syncthreads();
    }

    if (key >= m)
        return;
    E *kp = dk + (sp.begin + key) * gr.lddk + kvh * a.D, *vp = dv + (sp.begin + key) * gr.lddv + kvh * a.D;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
        store_col(kp, dka[d], 32 * d + 4 * h, a.D, a.scale);
        store_col(vp, dva[d], 32 * d + 4 * h, a.D, 1.f);
    }
}

template <typename E, int DC>
hipError_t launch(const E *q, const E *k, const E *v, const E *o, const float *lse, const E *dout,
                  E *dq, E *dk, E *dv, float *delta, AttnArgs a, const AttnGrads &gr,
                  hipStream_t st)
{
    constexpr bool F32 = sizeof(E) == 4;
    constexpr int NQ = 1, BK = F32 && DC > 64 ? 32 : 64, BR = !F32 && DC != 128 ? 64 : 32;
    AttnArgs b = a;
    a.slots = attn_slots(a.Tq, a.group.G, 128 * NQ, a.S);
    HEX_LAUNCH((attn_dq_k<E, DC, NQ, BK>), dim3(static_cast<uint32_t>(a.slots) * a.Hkv), dim3(256),
               0, st, q, k, v, o, lse, dout, dq, delta, a, gr);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    b.slots = attn_slots(a.Tk, 1, 128, a.S);
    HEX_LAUNCH((attn_dkv_k<E, DC, BR>), dim3(static_cast<uint32_t>(b.slots) * a.Hkv), dim3(256), 0,
               st, q, k, v, lse, dout, delta, dk, dv, b, gr);
    return hipGetLastError();
}

template <typename E>
hipError_t by_dim(const void *q, const void *k, const void *v, const void *o, const float *lse,
                  const void *dout, void *dq, void *dk, void *dv, float *delta, const AttnArgs &a,
                  const AttnGrads &gr, hipStream_t st)
{
    const auto run = [&](auto f) {
        return f(static_cast<const E *>(q), static_cast<const E *>(k), static_cast<const E *>(v),
                 static_cast<const E *>(o), lse, static_cast<const E *>(dout), static_cast<E *>(dq),
                 static_cast<E *>(dk), static_cast<E *>(dv), delta, a, gr, st);
    };
    if (a.D <= 32)
        return run(launch<E, 32>);
    if (a.D <= 64)
        return run(launch<E, 64>);
    if (a.D <= 96)
        return run(launch<E, 96>);
    return run(launch<E, 128>);
}

} // namespace
} // namespace attn

hipError_t attn_bwd(const void *q, const void *k, const void *v, const void *o, const float *lse,
                    const void *dout, void *dq, void *dk, void *dv, float *delta,
                    const AttnArgs &a, const AttnGrads &gr, Dtype dt, hipStream_t st)
{
    return dt == F32
               ? attn::by_dim<float>(q, k, v, o, lse, dout, dq, dk, dv, delta, a, gr, st)
               : attn::by_dim<bf16raw>(q, k, v, o, lse, dout, dq, dk, dv, delta, a, gr, st);
}

} // namespace hexk
