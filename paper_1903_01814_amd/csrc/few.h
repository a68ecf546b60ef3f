// few.h -- projections of a few tokens (serving: one or a few new tokens of every
// stream), D[m][n] = sum over k of x[m][k] w[n][k] with the epilogues of gemm.h.
//
// The time is that of reading the weights once, so all of them have to be on
// their way at once: a block takes 16 rows of w (or eight; GATED: and as many
// partners), its waves take chunks of 128 bytes of k in turn, four chunks' loads ahead, and
// add their sums in LDS at the end, in the waves' order.  No workspace, nothing
// laid out before: float32 is multiplied as it is, and rows of any alignment are
// read as they lie.
//
// A load takes eight rows of 128 bytes (whole cache lines); a wave's own piece of
// LDS, 16-byte chunks permuted by the row, turns that into operands of 16 x 16
// products (bfloat16 32 k, float32 4), weights as the rows.  Tokens go in groups
// of 16; rows past the last token are zeros.
//
// bfloat16, four tokens: 2048 x 2048 (8.4 MB) 5.0 us, 2 x 5464 x 2048 (45 MB) 11.9 (3.8
// TB/s), 2048 x 5464 (22 MB) 7.2; the launch and the first load are 3 of each.
#pragma once

#include "act.h"
#include "attn.h"

namespace hexk {
namespace few {

typedef float floatx4 __attribute__((ext_vector_type(4)));

// Up to so many tokens.  Each 16 of them read x once more for every 16 rows of w,
// from the cache (bfloat16, 2048 x 5464, 32 tokens: 10.9 us, the tiles of gemm.h 11.9 and
// more; 4 tokens of 2048 x 2048: 4.9 against 11.9).
constexpr int kMost = 32;

struct Args {
    const void *w, *x;
    int64_t ldx;
    int M, N, K;
    int half; // gated: rows of w between a gate's row and its partner's
};

// 16 bytes of a row, n elements of it before its end (zeros behind)
template <typename E, bool VEC> __device__ __forceinline__ uint4 load16(const E *p, int n)
{
    constexpr int V = 16 / sizeof(E);
    uint4 u{0, 0, 0, 0};
    if (VEC) {
        if (n > 0) // whole vectors
            u = *reinterpret_cast<const uint4 *>(p);
    } else if (n >= V) {
        __builtin_memcpy(&u, p, 16);
    } else if (n > 0) {
        E v[V];
#pragma unroll
        for (int i = 0; i < V; ++i)
            v[i] = i < n ? p[i] : E(0);
        __builtin_memcpy(&u, v, 16);
    }
    return u;
}

__device__ __forceinline__ floatx4 multiply(const uint4 &a, const uint4 &b, floatx4 c, bf16raw)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(attn::bf16x8, a),
                                                   __builtin_bit_cast(attn::bf16x8, b), c, 0, 0, 0);
}
// lane l holds k = 4 (l / 16) + i of 16: four products, one i each
__device__ __forceinline__ floatx4 multiply(const uint4 &a, const uint4 &b, floatx4 c, float)
{
    const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[i]), __uint_as_float(y[i]), c, 0,
                                                 0, 0);
    return c;
}

// WR and XR: loads of eight rows of w (1 or 2) and of x (1, 2, 4).  Half the rows a
// block, half of the product's then unused, where there would not be a block for
// every compute unit otherwise (4 x 2048 x 2048: 5.7 -> 4.9 us, 4 x 2048 x 5464 8.4 ->
// 7.6).
template <typename E, int WR, int XR, bool GATED, bool VEC, typename Epi>
__global__ __launch_bounds__(GATED ? 512 : 1024) void few_k(Args a, Epi e)
{
    constexpr int V = 16 / sizeof(E), KC = 8 * V; // k of a vector, of a chunk
    constexpr int H = GATED ? 2 : 1, TG = (XR + 1) / 2;
    constexpr int R = H + TG, L = H * WR + XR;    // pieces of 16 rows x 128 bytes; loads
    constexpr int U = L <= 3 ? 4 : L <= 6 ? 3 : 2; // chunks' loads under way
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int n0 = blockIdx.x * (8 * WR);
    char *mine = lds + wave * (R * 2048);

    // this lane's row and place in LDS of each load, its vector of the chunks
    const int lr = lane >> 3, lc = lane & 7;
    auto at = [&](int piece, int r, int c) {
        return reinterpret_cast<uint4 *>(mine + piece * 2048 + r * 128 + ((c ^ (r >> 1 & 7)) << 4));
    };
    const E *row[L];
    bool live[L];
    uint4 *to[L];
#pragma unroll
    for (int l = 0; l < L; ++l) {
        if (l < H * WR) {
            const int h = l / WR, r = lr + 8 * (l % WR), n = min(n0 + r, a.N - 1);
            row[l] = static_cast<const E *>(a.w) + static_cast<int64_t>(n + h * a.half) * a.K;
            live[l] = true;
            to[l] = at(h, r, lc);
        } else {
            const int x = l - H * WR, m = lr + 8 * x;
            live[l] = m < a.M;
            row[l] = static_cast<const E *>(a.x) + (m < a.M ? m : 0) * a.ldx;
            to[l] = at(H + x / 2, lr + 8 * (x % 2), lc);
        }
    }
    const int chunks = (a.K + KC - 1) / KC;

    floatx4 acc[H][TG] = {};
    for (int c0 = wave; c0 < chunks; c0 += waves * U) {
        uint4 u[U][L];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int k = (c0 + j * waves) * KC + lc * V;
#pragma unroll
            for (int l = 0; l < L; ++l)
                u[j][l] = live[l] ? load16<E, VEC>(row[l] + (k < a.K ? k : 0), a.K - k)
                                  : uint4{0, 0, 0, 0};
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (c0 + j * waves >= chunks)
                break;
#pragma unroll
            for (int l = 0; l < L; ++l)
                *to[l] = u[j][l];
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                // rows that no load wrote: what lies there, in results that are not used
                const int r = lane & 15, c = 4 * s + (lane >> 4);
                uint4 f[R];
#pragma unroll
                for (int p = 0; p < R; ++p)
                    f[p] = *at(p, r, c);
#pragma unroll
                for (int h = 0; h < H; ++h)
#pragma unroll
                    for (int g = 0; g < TG; ++g)
                        acc[h][g] = multiply(f[h], f[H + g], acc[h][g], E{});
            }
            __builtin_amdgcn_wave_barrier();
        }
    }

    // [wave][h][g][token][16 n]
    __syncthreads();
    float *sums = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int g = 0; g < TG; ++g)
            *reinterpret_cast<floatx4 *>(sums + ((wave * H + h) * TG + g) * 256 +
                                         (lane & 15) * 16 + 4 * (lane >> 4)) = acc[h][g];
    __syncthreads();
    // a thread eight columns of a token
    const int t = threadIdx.x / WR % 16, g = threadIdx.x / (16 * WR), m = 16 * g + t;
    const int n = n0 + 8 * (threadIdx.x % WR);
    if (g >= TG || m >= a.M || n >= a.N)
        return;
    const auto cols = e.cols(n);
    const auto f = e.fetch(m, n);
    float v[H][8] = {};
    for (int w = 0; w < waves; ++w)
#pragma unroll
        for (int h = 0; h < H; ++h) {
            float x[8];
            row8<float, true>(sums + ((w * H + h) * TG + g) * 256 + t * 16 + (n - n0), 8, x);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[h][i] += x[i];
        }
    if constexpr (GATED)
        e.done(m, n, v[0], v[1], cols);
    else
        e.done(m, n, v[0], cols, f);
}

template <typename E, int WR, int XR, bool GATED, typename Epi>
hipError_t launch_for(const Args &a, const Epi &e, bool vec, hipStream_t st)
{
    const int blocks = (a.N + 8 * WR - 1) / (8 * WR);
    const int chunks = static_cast<int>((a.K * sizeof(E) + 127) / 128);
    // 16 waves where a compute unit has one block (4 x 2048 x 5464: 8.1 -> 7.8 us), eight
    // else, so that two blocks fit; none without a chunk
    int waves = GATED || blocks > device_cus() ? 8 : 16;
    while (waves > 1 && waves / 2 >= chunks)
        waves /= 2;
    const size_t lds = static_cast<size_t>(waves) * ((GATED ? 2 : 1) + (XR + 1) / 2) * 2048;
    if (vec)
        HEX_LAUNCH((few_k<E, WR, XR, GATED, true, Epi>), dim3(blocks), dim3(64 * waves), lds, st, a,
                   e);
    else
        HEX_LAUNCH((few_k<E, WR, XR, GATED, false, Epi>), dim3(blocks), dim3(64 * waves), lds, st,
                   a, e);
    return hipGetLastError();
}

template <typename E, int WR, bool GATED, typename Epi>
hipError_t launch_rows(const Args &a, const Epi &e, hipStream_t st)
{
    constexpr int64_t V = 16 / sizeof(E);
    const bool vec = a.K % V == 0 && a.ldx % V == 0;
    return a.M <= 8    ? launch_for<E, WR, 1, GATED>(a, e, vec, st)
           : a.M <= 16 ? launch_for<E, WR, 2, GATED>(a, e, vec, st)
                       : launch_for<E, WR, 4, GATED>(a, e, vec, st);
}

// M up to kMost; rows of w and x of any alignment
template <typename E, bool GATED, typename Epi>
hipError_t launch(const Args &a, const Epi &e, hipStream_t st)
{
    return (a.N + 15) / 16 < device_cus() ? launch_rows<E, 1, GATED>(a, e, st)
                                          : launch_rows<E, 2, GATED>(a, e, st);
}

} // namespace few
} // namespace hexk
