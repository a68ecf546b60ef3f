// k_linear.hip -- projections: y = act(x w^T + b) + res, and their gradients.
//
//   z = x w^T + b,  y = act(z) + res
//   dz = dy act'(z),  dx = dz w,  dw = dz^T x,  db = sum over rows of dz
//
// Matrix products of gemm.h with their epilogues; what bounds them stands there.
// bfloat16 calls round z (where it is kept) and dz once to bfloat16, as operands
// of the products that follow; sums are float32.
#include "few.h"
#include "gemm.h"
#include "tokens.h"

namespace hexk {
namespace {

using gemm::Plan;
using gemm::Side;

struct Nothing {};

// y = act(v + bias) + res, z = v + bias
template <typename E, int ACT> struct LinearEpi {
    const E *bias, *res;
    E *y, *z;
    int64_t ldr, ldy;
    int N;
    bool vec; // N, ldr and ldy whole vectors
    static constexpr bool kSums = false;
    struct Cols {
        float b[8];
    };
    struct Fetched {
        float r[8];
    };
    __device__ __forceinline__ Cols cols(int n) const
    {
        Cols c = {};
        if (bias != nullptr)
            row8<E, true>(bias + n, N - n, c.b);
        return c;
    }
    __device__ __forceinline__ Fetched fetch(int m, int n) const
    {
        Fetched f = {};
        if (res == nullptr)
            return f;
        if (vec)
            row8<E, true>(res + m * ldr + n, 8, f.r);
        else
            row8<E, false>(res + m * ldr + n, N - n, f.r);
        return f;
    }
    __device__ __forceinline__ void done(int m, int n, float (&v)[8], const Cols &c,
                                         const Fetched &f) const
    {
        E *pz = z + static_cast<int64_t>(m) * N + n, *py = y + m * ldy + n;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] += c.b[i];
        if (z != nullptr) {
            if (vec)
                save_row8<E, true>(pz, 8, v);
            else
                save_row8<E, false>(pz, N - n, v);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = activate<sizeof(E) == 4>(v[i], ACT) + f.r[i];
        if (vec)
            save_row8<E, true>(py, 8, v);
        else
            save_row8<E, false>(py, N - n, v);
    }
};

// Whether a tensor of rows of n elements, ld apart, is an operand as it is
// (bfloat16, whole vectors); others are packed.
bool ready(int64_t n, int64_t ld, Dtype dt) { return dt == BF16 && n % 8 == 0 && ld % 8 == 0; }

} // namespace

// The operand of a tensor [rows][cols]: itself, or a place in the workspace and
// the job that fills it.
Side operand(const void *src, const void *z, int act, int rows, int cols, int64_t ld, Dtype dt,
             Halves map, Space &ws, PackJobs &jobs, bool copy)
{
    if (act == ACT_NONE && map.half == map.halfp && ready(cols, ld, dt) && !copy)
        return Side{static_cast<const bf16raw *>(src), ld, 0, rows};
    const int planes = dt == F32 ? 3 : 1;
    const int64_t dld = pitch(cols);
    const int64_t drows = map.half > 0 ? 2 * static_cast<int64_t>(map.halfp) : rows;
    bf16raw *dst = ws.take<bf16raw>(planes * drows * dld);
    PackJob &q = jobs.job[jobs.n++];
    q = PackJob{src, z, dst, ld, dld, drows * dld, drows, rows, cols, map.half, map.halfp, act, 0};
    return Side{dst, dld, drows * dld, static_cast<int>(drows)};
}
// the same tensor read along its rows of memory: its columns are the operand's
Side tall(const Side &s, int cols)
{
    Side t = s;
    t.rows = static_cast<int>(round8(cols));
    return t;
}

namespace {

// y = v in O; rows may skip those between two halves.  SUMS: sums of the rows'
// operand to `sums`.
template <typename O, bool SUMS> struct StoreEpi {
    O *y, *sums;
    int64_t ldy;
    int N;
    Halves map;
    bool vec;
    static constexpr bool kSums = SUMS;
    struct Fetched {};
    __device__ __forceinline__ Nothing cols(int) const { return Nothing{}; }
    __device__ __forceinline__ Fetched fetch(int, int) const { return Fetched{}; }
    __device__ __forceinline__ void done(int m, int n, float (&v)[8], Nothing, Fetched) const
    {
        const int row = map.row(m);
        if (row < 0)
            return;
        O *p = y + row * ldy + n;
        if (vec)
            save_row8<O, true>(p, 8, v);
        else
            save_row8<O, false>(p, N - n, v);
    }
    __device__ __forceinline__ void sum(int m, float v) const
    {
        const int row = map.row(m);
        if (row >= 0)
            sums[row] = from_f<O>(v);
    }
};

template <int PL, typename O>
hipError_t store_as(bool tall_q, const Plan &pl, const Side &P, const Side &Q, float *ws, O *y,
                    int64_t ldy, O *sums, Halves map, hipStream_t st)
{
    const bool vec = pl.N % 8 == 0 && ldy % (16 / static_cast<int64_t>(sizeof(O))) == 0;
    if (tall_q && sums != nullptr)
        return gemm::launch<PL, true, true, false>(
            pl, P, Q, 0, ws, StoreEpi<O, true>{y, sums, ldy, pl.N, map, vec}, st);
    const StoreEpi<O, false> e{y, nullptr, ldy, pl.N, map, vec};
    if (tall_q)
        return gemm::launch<PL, true, true, false>(pl, P, Q, 0, ws, e, st);
    if constexpr (PL == 1 && sizeof(O) == 4) // weights' gradients alone have another type
        return hipErrorInvalidValue;
    else
        return gemm::launch<PL, true, false, false>(pl, P, Q, 0, ws, e, st);
}

} // namespace

// D = Q P stored as it is: Q wide (data gradient) or tall (weight gradient), P tall
hipError_t store_product(bool tall_q, const Plan &pl, const Side &P, const Side &Q, float *ws,
                         void *y, int64_t ldy, void *sums, Halves map, Dtype dt, hipStream_t st)
{
    float *yf = static_cast<float *>(y), *sf = static_cast<float *>(sums);
    if (pl.planes == 3) // float32 operands have float32 results
        return dt == F32 ? store_as<3>(tall_q, pl, P, Q, ws, yf, ldy, sf, map, st)
                         : hipErrorInvalidValue;
    return dt == F32 ? store_as<1>(tall_q, pl, P, Q, ws, yf, ldy, sf, map, st)
                     : store_as<1>(tall_q, pl, P, Q, ws, static_cast<bf16raw *>(y), ldy,
                                   static_cast<bf16raw *>(sums), map, st);
}

namespace {

template <typename E, int ACT>
LinearEpi<E, ACT> epilogue(const Output &o, int N)
{
    constexpr int64_t per = 16 / sizeof(E);
    const bool vec = N % 8 == 0 && o.ldr % per == 0 && o.ldy % per == 0;
    return LinearEpi<E, ACT>{static_cast<const E *>(o.bias), static_cast<const E *>(o.res),
                             static_cast<E *>(o.y), static_cast<E *>(o.z), o.ldr, o.ldy, N, vec};
}

template <typename E, int ACT>
hipError_t product_of(const Plan &pl, const Side &W, const Side &X, float *ws, const Output &o,
                      hipStream_t st)
{
    return gemm::launch<sizeof(E) == 4 ? 3 : 1, false, false, false>(
        pl, W, X, 0, ws, epilogue<E, ACT>(o, pl.N), st);
}
template <typename E, int ACT>
hipError_t few_of(const few::Args &a, const Output &o, hipStream_t st)
{
    return few::launch<E, false>(a, epilogue<E, ACT>(o, a.N), st);
}

} // namespace

hipError_t linear_product(const Plan &pl, const Side &W, const Side &X, float *ws, const Output &o,
                          int act, Dtype dt, hipStream_t st)
{
    return HEX_BY_TYPE(product_of, pl, W, X, ws, o, st);
}

hipError_t linear_few(const void *w, const void *x, int64_t ldx, int M, int N, int K,
                      const Output &o, int act, Dtype dt, hipStream_t st)
{
    const few::Args a{w, x, ldx, M, N, K, 0};
    return HEX_BY_TYPE(few_of, a, o, st);
}

size_t linear_fwd(const LinearArgs &a, void *ws, bool run, Dtype dt, hipStream_t st,
                  hipError_t &err)
{
    const Output o{a.bias, a.res, a.y, a.z, a.ldr, a.ldy};
    if (a.M <= few::kMost) {
        if (run)
            err = linear_few(a.w, a.x, a.ldx, a.M, a.N, a.K, o, a.act, dt, st);
        return 0;
    }
    Space sp{static_cast<char *>(ws)};
    PackJobs jobs{};
    const Side X = operand(a.x, nullptr, 0, a.M, a.K, a.ldx, dt, Halves{0, 0}, sp, jobs);
    const Side W = operand(a.w, nullptr, 0, a.N, a.K, a.K, dt, Halves{0, 0}, sp, jobs);
    const Plan pl = gemm::make_plan(a.M, a.N, a.K, false, dt == F32 ? 3 : 1);
    float *part = sp.take<float>(gemm::part_bytes(pl, false) / 4);
    if (run && (err = pack(jobs, dt, st)) == hipSuccess)
        err = linear_product(pl, W, X, part, o, a.act, dt, st);
    return sp.used;
}

size_t linear_bwd(const LinearArgs &a, const LinearGrads &g, void *ws, bool run, Dtype dt,
                  hipStream_t st, hipError_t &err)
{
    // all places are taken whatever is asked for, so that one size does
    const int planes = dt == F32 ? 3 : 1;
    const Halves none{0, 0};
    Space sp{static_cast<char *>(ws)};
    PackJobs dzj{}, xj{}, wj{};
    const Side DZ = operand(g.dy, a.z, a.act, a.M, a.N, g.lddy, dt, none, sp, dzj);
    const Side X = operand(a.x, nullptr, 0, a.M, a.K, a.ldx, dt, none, sp, xj);
    const Side W = operand(a.w, nullptr, 0, a.N, a.K, a.K, dt, none, sp, wj);
    const Plan px = gemm::make_plan(a.M, a.K, a.N, false, planes);
    const Plan pw = gemm::make_plan(a.N, a.K, a.M, false, planes);
    const size_t part = gemm::part_bytes(px, false), partw = gemm::part_bytes(pw, false);
    float *parts = sp.take<float>((part > partw ? part : partw) / 4);
    float *sums = sp.take<float>(static_cast<int64_t>(col_sum_slices(a.M, a.N)) * a.N);
    if (!run)
        return sp.used;
    PackJobs jobs{};
    for (const PackJobs *j : {&dzj, g.dw != nullptr ? &xj : nullptr, g.dx != nullptr ? &wj : nullptr})
        if (j != nullptr && j->n > 0)
            jobs.job[jobs.n++] = j->job[0];
    if ((err = pack(jobs, dt, st)) != hipSuccess)
        return sp.used;
    if (g.dx != nullptr && (err = store_product(false, px, tall(W, a.K), DZ, parts, g.dx, g.lddx,
                                                nullptr, none, dt, st)) != hipSuccess)
        return sp.used;
    // db beside dw where that product can give it
    const bool beside = g.dw != nullptr && gemm::gives_sums(pw);
    if (g.dw != nullptr &&
        (err = store_product(true, pw, tall(X, a.K), tall(DZ, a.N), parts, g.dw, a.K,
                             beside ? g.db : nullptr, none, g.dwt, st)) != hipSuccess)
        return sp.used;
    if (g.db != nullptr && !beside) {
        if (dzj.n > 0)
            err = col_sum(DZ.p, DZ.ld, DZ.plane, planes, a.M, a.N, none, sums, g.db, BF16, g.dwt, st);
        else
            err = col_sum(g.dy, g.lddy, 0, 1, a.M, a.N, none, sums, g.db, dt, g.dwt, st);
    }
    return sp.used;
}

} // namespace hexk
