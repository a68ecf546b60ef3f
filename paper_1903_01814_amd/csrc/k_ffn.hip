// k_ffn.hip -- the gated feed-forward block and its gradients.
//
//   g = x wg^T + bg,  u = x wu^T + bu,  h = act(g) u,  y = h w2^T + b2 + res
//   dh = dy w2,  dg = dh u act'(g),  du = dh act(g)
//   dx = [dg du] [wg; wu],  dw1 = [dg du]^T x,  dw2 = dy^T h
//
// Both projections are one product whose waves hold a column of the gate and of
// its partner in the same lane, so h is made in its epilogue; dg and du are made
// in the epilogue of dh's product, and dh never reaches memory.  bfloat16 calls
// round h, dg and du once to bfloat16, as operands of the products that follow, and g
// and u where they are kept for the backward (below); h is made of unrounded ones.
//
// 16432 tokens, 2048 to 5464 to 2048 features, bfloat16: g, u and h 765 us (961
// TFLOP/s), dg and du 564 (their product, 1.3 GB of g, u, dg and du besides), the
// others as gemm.h says.  Made apart from its product, h would take another pass over g
// and u, 0.36 GB.
#include "few.h"
#include "gemm.h"
#include "tokens.h"

namespace hexk {
namespace {

using gemm::Plan;
using gemm::Side;

// ---- how g and u are kept for the backward: float32 as they are; bfloat16 calls
// have 16 bits a value.  With bfloat16's 8 bits of precision there, dx and dw1
// would carry three roundings of like size (g and u, dg and du, the result: 3.0e-3
// of their norm); so eight values in a row become float16, 11 bits, where all of
// them have its exponents, 2^-14 .. 2^15, and bfloat16 where one has not: 2.4e-3,
// as a projection's gradients have.  The first value's last bit says which (1:
// float16), so that it is off by up to a step of its type, twice a rounding.
struct Kept {
    template <typename E> static __device__ __forceinline__ void save(E *p, const float (&v)[8])
    {
        if constexpr (sizeof(E) == 4) {
            save_row8<E, true>(p, 8, v);
        } else {
            float most = fabsf(v[0]), least = fabsf(v[0]);
#pragma unroll
            for (int i = 1; i < 8; ++i) {
                most = fmaxf(most, fabsf(v[i]));
                least = fminf(least, fabsf(v[i]));
            }
            // a NaN is not seen by the two, but by the sum
            float nan = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                nan += 0.f * v[i];
            uint4 u;
            if (most < 32768.f && least >= 6.103515625e-5f && nan == 0.f) {
                half8 h;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    h[i] = static_cast<_Float16>(v[i]);
                u = __builtin_bit_cast(uint4, h);
                // the first cut, not rounded: the odd number that it lies next to is then
                // a step away at most, half a step more after rounding
                const uint32_t cut =
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(v[0], 0.f));
                u.x = (u.x & 0xffff0000u) | (cut & 0xffffu) | 1u;
            } else {
                pack8<bf16raw>(v, &u);
                // the first to 7 bits, to nearest even
                const uint32_t b = __float_as_uint(v[0]);
                const uint32_t r = v[0] != v[0] ? 0x7fc0u : (b + 0xffffu + (b >> 17 & 1u)) >> 17 << 1;
                u.x = (u.x & 0xffff0000u) | r;
            }
            *reinterpret_cast<uint4 *>(p) = u;
        }
    }
    template <typename E> static __device__ __forceinline__ void load(const E *p, float (&v)[8])
    {
        if constexpr (sizeof(E) == 4) {
            row8<E, true>(p, 8, v);
        } else {
            const uint4 u = *reinterpret_cast<const uint4 *>(p);
            if (u.x & 1u) {
                const half8 h = __builtin_bit_cast(half8, u);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = static_cast<float>(h[i]);
            } else {
                unpack8<bf16raw>(&u, v);
            }
        }
    }

  private:
    typedef _Float16 half8 __attribute__((ext_vector_type(8)));
};

// g + bg, u + bu to gu (nullable), h = act(g) u; zeros in the columns F .. Fp - 1
template <typename E, int ACT> struct GatedEpi {
    const E *bias; // bg, then bu
    E *gu, *h;
    int64_t Fp;
    int F;
    static constexpr bool kSums = false;
    struct Cols {
        float g[8], u[8];
    };
    struct Fetched {};
    __device__ __forceinline__ Cols cols(int f) const
    {
        Cols c = {};
        if (bias != nullptr) {
            row8<E, false>(bias + f, F - f, c.g);
            row8<E, false>(bias + F + f, F - f, c.u);
        }
        return c;
    }
    __device__ __forceinline__ Fetched fetch(int, int) const { return Fetched{}; }
    __device__ __forceinline__ void done(int m, int f, float (&g)[8], float (&u)[8],
                                         const Cols &c) const
    {
        constexpr bool FINE = sizeof(E) == 4;
        constexpr float zeros[8] = {};
        const int k = F - f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            g[i] += c.g[i];
            u[i] += c.u[i];
        }
        if (k < 8)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                g[i] = i < k ? g[i] : 0.f;
                u[i] = i < k ? u[i] : 0.f;
            }
        if (gu != nullptr) {
            E *p = gu + static_cast<int64_t>(m) * 2 * Fp + f;
            Kept::save(p, g);
            Kept::save(p + Fp, u);
            if (k <= 8)
                for (int64_t c = 8; c < Fp - f; c += 8) {
                    save_row8<E, true>(p + c, 8, zeros);
                    save_row8<E, true>(p + Fp + c, 8, zeros);
                }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            g[i] = activate<FINE>(g[i], ACT) * u[i];
        if (k < 8) // act(0) u = 0 but for the sign
#pragma unroll
            for (int i = 0; i < 8; ++i)
                g[i] = i < k ? g[i] : 0.f;
        E *p = h + static_cast<int64_t>(m) * Fp;
        save_row8<E, true>(p + f, 8, g);
        if (k <= 8)
            for (int64_t c = f + 8; c < Fp; c += 8)
                save_row8<E, true>(p + c, 8, zeros);
    }
};

// dg and du from dh, in bfloat16 or in three planes, side by side; in the columns
// from F to a whole vector dh, g and u are zeros, so dg and du are
template <typename E, int ACT> struct GatedGradEpi {
    const E *gu;
    bf16raw *d;
    int64_t Fp, F8, ldd, plane; // columns of half of gu, of d; rows of d
    static constexpr bool kSums = false;
    struct Nothing {};
    struct Fetched {
        float g[8], u[8];
    };
    __device__ __forceinline__ Nothing cols(int) const { return Nothing{}; }
    __device__ __forceinline__ Fetched fetch(int m, int f) const
    {
        Fetched x;
        const E *p = gu + static_cast<int64_t>(m) * 2 * Fp + f;
        Kept::load(p, x.g);
        Kept::load(p + Fp, x.u);
        return x;
    }
    __device__ __forceinline__ void done(int m, int f, float (&dh)[8], Nothing,
                                         const Fetched &x) const
    {
        constexpr bool FINE = sizeof(E) == 4;
        const int64_t at = static_cast<int64_t>(m) * ldd + f;
        float dg[8], du[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float a;
            const float s = derivative<FINE>(x.g[i], ACT, a);
            dg[i] = dh[i] * x.u[i] * s;
            du[i] = dh[i] * a;
        }
        if constexpr (FINE) {
            save_planes(d + at, plane, dg);
            save_planes(d + at + F8, plane, du);
        } else {
            save_row8<bf16raw, true>(d + at, 8, dg);
            save_row8<bf16raw, true>(d + at + F8, 8, du);
        }
    }
};

template <typename E, int ACT> GatedEpi<E, ACT> gated(const FfnArgs &a)
{
    return GatedEpi<E, ACT>{static_cast<const E *>(a.b1), static_cast<E *>(a.gu),
                            static_cast<E *>(a.h), pitch(a.F), a.F};
}
template <typename E, int ACT>
hipError_t gated_product(const Plan &pl, const Side &W, const Side &X, float *ws, const FfnArgs &a,
                         hipStream_t st)
{
    return gemm::launch<sizeof(E) == 4 ? 3 : 1, false, false, true>(
        pl, W, X, static_cast<int>(round8(a.F)), ws, gated<E, ACT>(a), st);
}
template <typename E, int ACT> hipError_t gated_few(const FfnArgs &a, hipStream_t st)
{
    return few::launch<E, true>(few::Args{a.w1, a.x, a.ldx, a.M, a.F, a.K, a.F}, gated<E, ACT>(a),
                                st);
}

template <typename E, int ACT>
hipError_t gated_grad(const Plan &pl, const Side &W2, const Side &DY, float *ws, const void *gu,
                      const Side &D, int F, hipStream_t st)
{
    return gemm::launch<sizeof(E) == 4 ? 3 : 1, true, false, false>(
        pl, W2, DY, 0, ws,
        GatedGradEpi<E, ACT>{static_cast<const E *>(gu), const_cast<bf16raw *>(D.p), pitch(F),
                             round8(F), D.ld, D.plane},
        st);
}

} // namespace

int ffn_width(int F) { return static_cast<int>(pitch(F)); }

// From so many tokens on w2 is copied to rows that begin on cache lines, as h's do.
// Forward in us, without and with the copy:
//   features          4096 tokens     8192           12288          16384
//   512 and 1368      36.4    38.6    59.8    61.6   88.9    90.5   104.5   104.0
//   1024 and 2736     97.1   100.3   168.6   168.4   252.9   250.1  294.1   295.0
//   2048 and 1368     96.4    97.4   159.0   160.9   234.5   234.4  275.5   279.2
//   1024 and 5464     165.9  168.7   343.0   330.7   487.5   465.9  570.7   549.4
//   2048 and 5464     303.4  295.0   506.1   507.4   799.5   791.8  1035.9  1000.6
// A copy costs 2 to 4 us where h is small beside the caches, and gains 1 to 4 % from
// where it is not; 32768 tokens of 2048 and 5464 2048 and 1970.
constexpr int kCopy = 8192;

size_t ffn_fwd(const FfnArgs &a, void *ws, bool run, Dtype dt, hipStream_t st, hipError_t &err)
{
    const int act = a.act, planes = dt == F32 ? 3 : 1;
    const int64_t Fp = pitch(a.F);
    const Output o{a.b2, a.res, a.y, nullptr, a.ldr, a.ldy};
    if (a.M <= few::kMost) {
        if (run && (err = HEX_BY_TYPE(gated_few, a, st)) == hipSuccess)
            err = linear_few(a.w2, a.h, Fp, a.M, a.N, a.F, o, ACT_NONE, dt, st);
        return 0;
    }
    const Halves none{0, 0}, halves{a.F, static_cast<int>(round8(a.F))};
    Space sp{static_cast<char *>(ws)};
    PackJobs jobs{}, late{};
    const Side X = operand(a.x, nullptr, 0, a.M, a.K, a.ldx, dt, none, sp, jobs);
    const Side W1 = operand(a.w1, nullptr, 0, 2 * a.F, a.K, a.K, dt, halves, sp, jobs);
    const bool copy = a.M >= kCopy && a.F != pitch(a.F);
    const Side W2 = operand(a.w2, nullptr, 0, a.N, a.F, a.F, dt, none, sp, jobs, copy);
    const Side H = operand(a.h, nullptr, 0, a.M, static_cast<int>(Fp), Fp, dt, none, sp, late);
    const Plan p1 = gemm::make_plan(a.M, a.F, a.K, true, planes);
    const Plan p2 = gemm::make_plan(a.M, a.N, a.F, false, planes);
    const size_t b1 = gemm::part_bytes(p1, true), b2 = gemm::part_bytes(p2, false);
    float *part = sp.take<float>((b1 > b2 ? b1 : b2) / 4);
    if (run && (err = pack(jobs, dt, st)) == hipSuccess &&
        (err = HEX_BY_TYPE(gated_product, p1, W1, X, part, a, st)) == hipSuccess &&
        (err = pack(late, dt, st)) == hipSuccess)
        err = linear_product(p2, W2, H, part, o, ACT_NONE, dt, st);
    return sp.used;
}

size_t ffn_bwd(const FfnArgs &a, const FfnGrads &g, void *ws, bool run, Dtype dt, hipStream_t st,
               hipError_t &err)
{
    const int planes = dt == F32 ? 3 : 1;
    const int64_t Fp = pitch(a.F);
    const int F8 = static_cast<int>(round8(a.F)), W = 2 * F8;
    const Halves none{0, 0}, halves{a.F, F8};
    Space sp{static_cast<char *>(ws)};
    PackJobs dyj{}, w2j{}, w1j{}, xj{}, hj{};
    const Side DY = operand(g.dy, nullptr, 0, a.M, a.N, g.lddy, dt, none, sp, dyj);
    const Side W2 = operand(a.w2, nullptr, 0, a.N, a.F, a.F, dt, none, sp, w2j);
    const Side W1 = operand(a.w1, nullptr, 0, 2 * a.F, a.K, a.K, dt, halves, sp, w1j);
    const Side X = operand(a.x, nullptr, 0, a.M, a.K, a.ldx, dt, none, sp, xj);
    const Side H = operand(a.h, nullptr, 0, a.M, static_cast<int>(Fp), Fp, dt, none, sp, hj);
    const int64_t ldd = pitch(W), plane = a.M * ldd;
    const Side D{sp.take<bf16raw>(planes * plane), ldd, plane, a.M};
    const Plan ph = gemm::make_plan(a.M, a.F, a.N, false, planes);
    const Plan px = gemm::make_plan(a.M, a.K, W, false, planes);
    const Plan p1 = gemm::make_plan(W, a.K, a.M, false, planes);
    const Plan p2 = gemm::make_plan(a.N, a.F, a.M, false, planes);
    size_t most = 0;
    for (const Plan *p : {&ph, &px, &p1, &p2})
        most = gemm::part_bytes(*p, false) > most ? gemm::part_bytes(*p, false) : most;
    float *part = sp.take<float>(most / 4);
    const int64_t sums1 = static_cast<int64_t>(col_sum_slices(a.M, W)) * W;
    const int64_t sums2 = static_cast<int64_t>(col_sum_slices(a.M, a.N)) * a.N;
    float *sums = sp.take<float>(sums1 > sums2 ? sums1 : sums2);
    if (!run)
        return sp.used;
    // dg and du are needed for all but dw2 and db2
    const bool inner = g.dx != nullptr || g.dw1 != nullptr || g.db1 != nullptr;
    PackJobs jobs{}, more{};
    auto add = [](PackJobs &to, const PackJobs &j, bool wanted) {
        if (wanted && j.n > 0)
            to.job[to.n++] = j.job[0];
    };
    add(jobs, dyj, inner || g.dw2 != nullptr);
    add(jobs, w2j, inner);
    add(jobs, w1j, g.dx != nullptr);
    add(jobs, xj, g.dw1 != nullptr);
    add(more, hj, g.dw2 != nullptr);
    if ((err = pack(jobs, dt, st)) != hipSuccess || (err = pack(more, dt, st)) != hipSuccess)
        return sp.used;
    const int act = a.act;
    if (inner && (err = HEX_BY_TYPE(gated_grad, ph, tall(W2, a.F), DY, part, a.gu, D, a.F, st)) !=
                     hipSuccess)
        return sp.used;
    if (g.dx != nullptr && (err = store_product(false, px, tall(W1, a.K), D, part, g.dx, g.lddx,
                                                nullptr, none, dt, st)) != hipSuccess)
        return sp.used;
    // the biases' gradients beside the weights' where those products can give them
    const bool beside1 = g.dw1 != nullptr && gemm::gives_sums(p1);
    const bool beside2 = g.dw2 != nullptr && gemm::gives_sums(p2);
    if (g.dw1 != nullptr &&
        (err = store_product(true, p1, tall(X, a.K), tall(D, W), part, g.dw1, a.K,
                             beside1 ? g.db1 : nullptr, halves, g.dwt, st)) != hipSuccess)
        return sp.used;
    if (g.dw2 != nullptr &&
        (err = store_product(true, p2, tall(H, a.F), tall(DY, a.N), part, g.dw2, a.F,
                             beside2 ? g.db2 : nullptr, none, g.dwt, st)) != hipSuccess)
        return sp.used;
    if (g.db1 != nullptr && !beside1 &&
        (err = col_sum(D.p, ldd, plane, planes, a.M, W, halves, sums, g.db1, BF16, g.dwt, st)) !=
            hipSuccess)
        return sp.used;
    if (g.db2 != nullptr && !beside2)
        err = col_sum(g.dy, g.lddy, 0, 1, a.M, a.N, none, sums, g.db2, dt, g.dwt, st);
    return sp.used;
}

} // namespace hexk
