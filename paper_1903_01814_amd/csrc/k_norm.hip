// k_norm.hip -- layer norm of rows, and its gradients.
//
//   n = (x - mean x) r,  r = 1 / sqrt(mean (x - mean x)^2 + eps),  y = n w + b
//   g = dy w,  dx = res + r (g - mean g - n mean (g n)),
//   dw = sum over rows of dy n,  db = sum over rows of dy
//
// Bound by memory: every element is read once and written once.  G lanes (8 to
// 64 of a wave, or a block of 256) keep a row in registers, 8 NV elements each,
// so the mean is taken before the deviations are squared, without a second
// read.  In the backward a block takes rows in turn and its lanes keep the sums
// of their own columns' dw and db; the blocks' sums are added by a second kernel
// in a fixed order.
#include "act.h"

namespace hexk {
namespace {

constexpr int kThreads = 256;

// sum over the G lanes of a row (G = 256: the block, through LDS); `turn`
// alternates two places in LDS, so that one barrier a sum is enough
template <int G, int N> __device__ __forceinline__ void row_sum(float (&s)[N], float *lds, int &turn)
{
#pragma unroll
    for (int o = (G < 64 ? G : 64) / 2; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i)
            s[i] += __shfl_xor(s[i], o);
    if constexpr (G > 64) {
        float *p = lds + turn * 8;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i)
                p[(threadIdx.x >> 6) * 2 + i] = s[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i)
            s[i] = (p[i] + p[2 + i]) + (p[4 + i] + p[6 + i]);
    }
}

// Columns of lane `l` of a row: vector j holds 8 (l + G j) .., n of them exist.
template <int G> __device__ __forceinline__ int col_of(int l, int j) { return 8 * (l + G * j); }

template <typename E, int G, int NV, bool VEC>
__global__ __launch_bounds__(kThreads) void norm_fwd_k(const E *x, const E *w, const E *b, E *y,
                                                       float *mean, float *rstd, NormArgs a)
{
    __shared__ float lds[16];
    int turn = 0;
    const int l = threadIdx.x % G;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads / G) + threadIdx.x / G;
    const bool live = row < a.T;
    const E *xr = x + (live ? row : 0) * a.ldx;
    float v[NV][8], s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = col_of<G>(l, j);
        row8<E, VEC>(xr + (c < a.C ? c : 0), a.C - c, v[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            s[0] += v[j][i];
    }
    row_sum<G>(s, lds, turn);
    const float mu = s[0] * a.inv;
    s[0] = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[j][i] -= mu;
            s[0] += col_of<G>(l, j) + i < a.C ? v[j][i] * v[j][i] : 0.f;
        }
    row_sum<G>(s, lds, turn);
    const float r = 1.f / sqrtf(fmaf(s[0], a.inv, a.eps));
    if (!live)
        return;
    if (l == 0 && mean != nullptr) {
        mean[row] = mu;
        rstd[row] = r;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = col_of<G>(l, j);
        if (c >= a.C)
            break;
        float wv[8], bv[8] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            wv[i] = 1.f;
        if (w != nullptr)
            row8<E, true>(w + c, a.C - c, wv);
        if (b != nullptr)
            row8<E, true>(b + c, a.C - c, bv);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[j][i] = fmaf(v[j][i] * r, wv[i], bv[i]);
        save_row8<E, VEC>(y + row * a.ldy + c, a.C - c, v[j]);
    }
}

// Block b takes the rows b, b + blocks, .. of kThreads / G at a time.  part
// [blocks][2][C]: the blocks' sums of dw and db.
template <typename E, int G, int NV, bool VEC, bool SUMS>
__global__ __launch_bounds__(kThreads) void norm_bwd_k(const E *x, const E *w, const float *mean,
                                                       const float *rstd, const E *dy,
                                                       const E *res, E *dx, float *part,
                                                       NormArgs a)
{
    constexpr int R = kThreads / G; // rows at a time
    __shared__ float lds[16];
    __shared__ float sums[SUMS && R > 1 ? 2 * kThreads * 8 * NV : 1];
    int turn = 0;
    const int l = threadIdx.x % G, sub = threadIdx.x / G;
    float wv[NV][8];
    float dw[NV][8] = {}, db[NV][8] = {};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = col_of<G>(l, j);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            wv[j][i] = 1.f;
        if (w != nullptr && c < a.C)
            row8<E, true>(w + c, a.C - c, wv[j]);
    }
    // the next row's elements are on their way while this one is worked on (51200
    // rows of 1024, bfloat16: 130 -> 92 us, 4.6 TB/s); rows of more than 8192 leave no
    // registers for that
    struct Row {
        Raw8<E> x[NV], g[NV], add[NV];
        float mu, r;
    } next;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * R;
    auto load = [&](int64_t row) {
        const bool in = row < a.T;
        const int64_t at = in ? row : 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = col_of<G>(l, j), k = in ? a.C - c : 0, from = c < a.C ? c : 0;
            next.x[j] = raw8<E, VEC>(x + at * a.ldx + from, k);
            next.g[j] = raw8<E, VEC>(dy + at * a.ldy + from, k);
            next.add[j] = raw8<E, VEC>(res != nullptr ? res + at * a.ldr + from : x,
                                       res != nullptr ? k : 0);
        }
        next.mu = mean[at];
        next.r = rstd[at];
    };
    constexpr bool AHEAD = NV < 8;
    if (AHEAD)
        load(static_cast<int64_t>(blockIdx.x) * R + sub);
    for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * R; r0 < a.T; r0 += stride) {
        const int64_t row = r0 + sub;
        const bool live = row < a.T;
        const int64_t at = row;
        if (!AHEAD)
            load(row);
        float n[NV][8], g[NV][8];
        Raw8<E> extra[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            unpack8<E>(next.x[j].u, n[j]);
            unpack8<E>(next.g[j].u, g[j]);
            extra[j] = next.add[j];
        }
        const float mu = next.mu, r = next.r;
        if (AHEAD && r0 + stride < a.T)
            load(row + stride);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // dead rows and columns past the row: n is left out with dy
                const bool in = live && col_of<G>(l, j) + i < a.C;
                n[j][i] = in ? (n[j][i] - mu) * r : 0.f;
                if constexpr (SUMS) {
                    dw[j][i] = fmaf(g[j][i], n[j][i], dw[j][i]);
                    db[j][i] += g[j][i];
                }
                g[j][i] *= wv[j][i];
                s[0] += g[j][i];
                s[1] = fmaf(g[j][i], n[j][i], s[1]);
            }
        row_sum<G>(s, lds, turn);
        if (!live)
            continue;
        const float mg = s[0] * a.inv, mgn = s[1] * a.inv;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = col_of<G>(l, j);
            if (c >= a.C)
                break;
            float add[8];
            unpack8<E>(extra[j].u, add);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                add[i] = fmaf(r, g[j][i] - mg - n[j][i] * mgn, add[i]);
            save_row8<E, VEC>(dx + at * a.lddx + c, a.C - c, add);
        }
    }
    if constexpr (SUMS) {
        float *out = part + static_cast<size_t>(blockIdx.x) * 2 * a.C;
        if constexpr (R == 1) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = col_of<G>(l, j) + i;
                    if (c < a.C) {
                        out[c] = dw[j][i];
                        out[a.C + c] = db[j][i];
                    }
                }
        } else {
            // [R][2][8 NV G]
            constexpr int W = 8 * NV * G;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = col_of<G>(l, j) + i;
                    sums[(sub * 2) * W + c] = dw[j][i];
                    sums[(sub * 2 + 1) * W + c] = db[j][i];
                }
            __syncthreads();
            for (int c = threadIdx.x; c < 2 * W; c += kThreads) {
                const int which = c / W, col = c % W;
                if (col >= a.C)
                    continue;
                float t = 0.f;
                for (int k = 0; k < R; ++k)
                    t += sums[(k * 2 + which) * W + col];
                out[which * a.C + col] = t;
            }
        }
    }
}

// out[c] = sum over the slots of part[slot][c], 16 columns a block, 64 slots side
// by side and eight of each on their way (1024 slots of 2048 columns: 20.7 -> 5.2 us);
// columns up to C go to dw, the others to db (either may be null)
constexpr int kJoin = 1024;
__global__ __launch_bounds__(kJoin) void norm_join_k(const float *part, int slots, int C,
                                                     float *dw, float *db)
{
    __shared__ float lds[kJoin / 16][17];
    const int c = blockIdx.x * 16 + threadIdx.x % 16, sub = threadIdx.x / 16;
    float t = 0.f;
    if (c < 2 * C)
#pragma unroll 8
        for (int s = sub; s < slots; s += kJoin / 16)
            t += part[static_cast<size_t>(s) * 2 * C + c];
    lds[sub][threadIdx.x % 16] = t;
    __syncthreads();
    if (sub != 0 || c >= 2 * C)
        return;
    t = 0.f;
#pragma unroll
    for (int s = 0; s < kJoin / 16; ++s)
        t += lds[s][threadIdx.x % 16];
    if (c < C && dw != nullptr)
        dw[c] = t;
    if (c >= C && db != nullptr)
        db[c - C] = t;
}

enum Pass { FWD, BWD, BWD_SUMS };

template <typename E, bool VEC, Pass P, int G, int NV>
hipError_t launch_one(const void *x, const void *w, const void *b, void *y, float *mean,
                      float *rstd, const void *dy, const void *res, void *dx, float *part,
                      int blocks, const NormArgs &a, hipStream_t st)
{
    const E *X = static_cast<const E *>(x), *W = static_cast<const E *>(w);
    if constexpr (P == FWD)
        HEX_LAUNCH((norm_fwd_k<E, G, NV, VEC>), dim3(blocks), dim3(kThreads), 0, st, X, W,
                   static_cast<const E *>(b), static_cast<E *>(y), mean, rstd, a);
    else
        HEX_LAUNCH((norm_bwd_k<E, G, NV, VEC, P == BWD_SUMS>), dim3(blocks), dim3(kThreads), 0, st,
                   X, W, mean, rstd, static_cast<const E *>(dy), static_cast<const E *>(res),
                   static_cast<E *>(dx), part, a);
    return hipGetLastError();
}

// Lanes and vectors of a row, by its length: one vector of eight a lane up to a
// wave, two up to 1024, then a block.  Half the lanes with twice the vectors, and
// twice or four times the lanes, took in us, forward / backward:
//   65536 x 128, bfloat16     8.8 / 15.2, half  8.9 / 15.6, twice 13.0 / 19.5
//   51200 x 512              21.3 / 31.4, half 18.8 / 37.7, four times 49.6 / 70.9
//   51200 x 1024             39.0 / 76.1,                   four times 68.5 / 99.7
//   16384 x 2048             27.6 / 52.2, a wave 24.0 / 79.5
//   16384 x 2048, float32    47.4 / 88.7, a wave 58.6 / 103.6
// so bfloat16's forward takes half the lanes where that was the faster.
template <typename E, bool VEC, Pass P>
hipError_t launch(const void *x, const void *w, const void *b, void *y, float *mean, float *rstd,
                  const void *dy, const void *res, void *dx, float *part, int blocks,
                  const NormArgs &a, hipStream_t st)
{
#define HEX_NORM_CALL(G, NV)                                                                  \
    launch_one<E, VEC, P, G, NV>(x, w, b, y, mean, rstd, dy, res, dx, part, blocks, a, st)
    constexpr bool HALF = P == FWD && sizeof(E) == 2;
    if (a.C <= 64)
        return HEX_NORM_CALL(8, 1);
    if (a.C <= 128)
        return HEX_NORM_CALL(16, 1);
    if (a.C <= 256)
        return HEX_NORM_CALL((HALF ? 16 : 32), (HALF ? 2 : 1));
    if (a.C <= 512)
        return HEX_NORM_CALL((HALF ? 32 : 64), (HALF ? 2 : 1));
    if (a.C <= 1024)
        return HEX_NORM_CALL(64, 2);
    if (a.C <= 2048)
        return HEX_NORM_CALL((HALF ? 64 : 256), (HALF ? 4 : 1));
    if (a.C <= 4096)
        return HEX_NORM_CALL(256, 2);
    if (a.C <= 8192)
        return HEX_NORM_CALL(256, 4);
    return HEX_NORM_CALL(256, 8);
#undef HEX_NORM_CALL
}

// rows of a block at a time, 256 / G of launch
int rows_at_a_time(int C, bool half)
{
    if (half && C > 128)
        return C <= 256 ? 16 : C <= 512 ? 8 : C <= 2048 ? 4 : 1;
    return C <= 64 ? 32 : C <= 128 ? 16 : C <= 256 ? 8 : C <= 1024 ? 4 : 1;
}

template <typename E> bool rows_aligned(std::initializer_list<int64_t> lds)
{
    for (int64_t ld : lds)
        if (ld % (16 / static_cast<int64_t>(sizeof(E))) != 0)
            return false;
    return true;
}

template <typename E>
hipError_t fwd(const void *x, const void *w, const void *b, void *y, float *mean, float *rstd,
               const NormArgs &a, hipStream_t st)
{
    const int64_t R = rows_at_a_time(a.C, sizeof(E) == 2);
    const int blocks = static_cast<int>((a.T + R - 1) / R);
    if (rows_aligned<E>({a.ldx, a.ldy}))
        return launch<E, true, FWD>(x, w, b, y, mean, rstd, nullptr, nullptr, nullptr, nullptr,
                                    blocks, a, st);
    return launch<E, false, FWD>(x, w, b, y, mean, rstd, nullptr, nullptr, nullptr, nullptr,
                                 blocks, a, st);
}

template <typename E>
hipError_t bwd(const void *x, const void *w, const float *mean, const float *rstd, const void *dy,
               const void *res, void *dx, float *dw, float *db, float *part, const NormArgs &a,
               hipStream_t st)
{
    const bool sums = dw != nullptr || db != nullptr;
    const bool vec = rows_aligned<E>({a.ldx, a.ldy, a.ldr, a.lddx});
    const int blocks = norm_bwd_blocks(a.T, a.C);
    float *mu = const_cast<float *>(mean), *rs = const_cast<float *>(rstd);
    hipError_t e;
    if (sums)
        e = vec ? launch<E, true, BWD_SUMS>(x, w, nullptr, nullptr, mu, rs, dy, res, dx, part,
                                            blocks, a, st)
                : launch<E, false, BWD_SUMS>(x, w, nullptr, nullptr, mu, rs, dy, res, dx, part,
                                             blocks, a, st);
    else
        e = vec ? launch<E, true, BWD>(x, w, nullptr, nullptr, mu, rs, dy, res, dx, part, blocks, a,
                                       st)
                : launch<E, false, BWD>(x, w, nullptr, nullptr, mu, rs, dy, res, dx, part, blocks,
                                        a, st);
    if (e != hipSuccess || !sums)
        return e;
    HEX_LAUNCH((norm_join_k), dim3((2 * a.C + 15) / 16), dim3(kJoin), 0, st, part, blocks, a.C,
               dw, db);
    return hipGetLastError();
}

} // namespace

// Blocks of the backward, each of which leaves 2 C sums: four a compute unit,
// fewer where there are not four turns of rows for each.
int norm_bwd_blocks(int64_t T, int C)
{
    const int64_t R = rows_at_a_time(C, false), turns = (T + R - 1) / R;
    const int64_t most = 4 * static_cast<int64_t>(device_cus());
    int64_t n = (turns + 3) / 4;
    return static_cast<int>(n > most ? most : n);
}

hipError_t norm_fwd(const void *x, const void *w, const void *b, void *y, float *mean, float *rstd,
                    const NormArgs &a, Dtype dt, hipStream_t st)
{
    return dt == F32 ? fwd<float>(x, w, b, y, mean, rstd, a, st)
                     : fwd<bf16raw>(x, w, b, y, mean, rstd, a, st);
}

hipError_t norm_bwd(const void *x, const void *w, const float *mean, const float *rstd,
                    const void *dy, const void *res, void *dx, float *dw, float *db, void *ws,
                    const NormArgs &a, Dtype dt, hipStream_t st)
{
    float *part = static_cast<float *>(ws);
    return dt == F32 ? bwd<float>(x, w, mean, rstd, dy, res, dx, dw, db, part, a, st)
                     : bwd<bf16raw>(x, w, mean, rstd, dy, res, dx, dw, db, part, a, st);
}

// dw and db (where not null) := 0, by the join of no slots
hipError_t norm_zero(float *dw, float *db, int C, hipStream_t st)
{
    if (dw == nullptr && db == nullptr)
        return hipSuccess;
    HEX_LAUNCH((norm_join_k), dim3((2 * C + 15) / 16), dim3(kJoin), 0, st,
               static_cast<const float *>(nullptr), 0, C, dw, db);
    return hipGetLastError();
}

} // namespace hexk
