// k_rotary.hip -- norm of every query and key head and rotation by positions
// of several axes, one pass; the same with keys and values stored in their
// cache places; and the gradients.
//
//   n = x / sqrt(mean(x^2) + eps),  y = n w   (without the norm: y = x)
//   pair j = (y_j, y_(j + D/2)) turned by the angle pos[axis_j] freq_j
//
// Bound by memory: every element is read and written once (51200 tokens, 16 + 4
// heads of 64 in bfloat16: forward 58 us, 4.5 TB/s; backward 86, 4.6 TB/s; a
// large copy reaches 4.95).  A block takes up to kTokens tokens at a time, makes
// their cosines and sines once for all heads (LDS: some thirty instructions a
// pair, for Hq + Hkv heads), and a group of L lanes takes a head: four pairs a
// lane, two 8- or 16-byte loads, the head's sum of squares by exchanges within
// the group.  The backward adds the weights' gradients in registers over a
// block's tokens, then over the block in LDS, then over the blocks in
// rotary_reduce_k, always in the same order.
#include "hexdev.h"
#include "kernels.h"

namespace hexk {
namespace {

constexpr int kTokens = 8;

template <typename E> struct Vec4;
template <> struct Vec4<float> {
    using type = float4;
};
template <> struct Vec4<bf16raw> {
    using type = ushort4;
};

template <typename E> __device__ __forceinline__ void load4(const E *p, float (&x)[4])
{
    const auto u = *reinterpret_cast<const typename Vec4<E>::type *>(p);
    x[0] = to_f(u.x), x[1] = to_f(u.y), x[2] = to_f(u.z), x[3] = to_f(u.w);
}
template <typename E> __device__ __forceinline__ void save4(E *p, const float (&x)[4])
{
    typename Vec4<E>::type u;
    u.x = from_f<E>(x[0]), u.y = from_f<E>(x[1]), u.z = from_f<E>(x[2]), u.w = from_f<E>(x[3]);
    *reinterpret_cast<typename Vec4<E>::type *>(p) = u;
}

// cos and sin of p f.  The product is kept exactly as hi + lo, a multiple of
// pi/2 in three parts is taken off (each step one rounding, by fused
// multiply-add), and the rest, at most pi/4, goes into the Taylor sums (first
// term left out below 2e-9).  Good to 1e-7 for angles up to 2^20, where the
// plain product of two floats would already be off by 0.06.
__device__ __forceinline__ float2 turn(float p, float f)
{
    const float hi = p * f, lo = fmaf(p, f, -hi);
    const float n = rintf(hi * 0.636619772f);
    float r = fmaf(n, -1.57079637e+00f, hi); // pi/2 rounded to float, then what is left
    r = fmaf(n, 4.37113883e-08f, r);
    r = fmaf(n, 1.71512451e-15f, r);
    r += lo;
    const float z = r * r;
    const float s =
        fmaf(r * z,
             fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), r);
    const float c = fmaf(
        z,
        fmaf(z,
             fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f),
             -0.5f),
        1.f);
    const int k = static_cast<int>(n);
    const float a = k & 1 ? s : c, b = k & 1 ? c : s;
    return float2{(k + 1) & 2 ? -a : a, k & 2 ? -b : b};
}

// cosines and sines of a block's tokens, [tokens][D / 2]
__device__ __forceinline__ void make_turns(float2 *cs, const RotaryArgs &a, int64_t t0, int tokens)
{
    const int half = a.D / 2;
    for (int e = threadIdx.x; e < tokens * half; e += blockDim.x) {
        const int t = e / half, j = e - t * half;
        const int ax = a.axis[j];
        // an axis that does not exist turns nothing
        const bool ok = ax >= 0 && ax < a.A;
        cs[e] = ok ? turn(a.pos[(t0 + t) * a.A + ax], a.freq[j]) : float2{1.f, 0.f};
    }
}

template <int L> __device__ __forceinline__ float sum_lanes(float v)
{
#pragma unroll
    for (int d = 1; d < L; d <<= 1)
        v += __shfl_xor(v, d);
    return v;
}

// L lanes a head (D <= 8 L)
template <typename E, int L, bool NORM>
__global__ __launch_bounds__(256) void rotary_fwd_k(const E *q, const E *k, const E *v, const E *wq,
                                                    const E *wk, E *qo, E *ko, E *vo,
                                                    const int32_t *slot, RotaryArgs a, int per)
{
    __shared__ float2 cs[kTokens * 4 * L];
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * per;
    const int tokens = static_cast<int>(a.T - t0 < per ? a.T - t0 : per);
    const int half = a.D / 2;
    const int c = 4 * (threadIdx.x % L);
    const bool in = c < half;
    const int heads = a.Hq + a.Hkv + (vo != nullptr ? a.Hkv : 0);
    float wq1[4], wq2[4], wk1[4], wk2[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        wq1[i] = wq2[i] = wk1[i] = wk2[i] = 1.f;
    if (in && wq != nullptr) {
        load4(wq + c, wq1);
        load4(wq + half + c, wq2);
    }
    if (in && wk != nullptr) {
        load4(wk + c, wk1);
        load4(wk + half + c, wk2);
    }
    make_turns(cs, a, t0, tokens);
    __syncthreads();
    // every lane of a group runs the same turns
    for (int e = threadIdx.x / L; e < tokens * heads; e += 256 / L) {
        const int tt = e / heads, hd = e - tt * heads;
        const int64_t t = t0 + tt;
        const bool isq = hd < a.Hq, isv = hd >= a.Hq + a.Hkv;
        const E *src = isq ? q + t * a.ldq + hd * a.D
                           : (isv ? v + t * a.ldv + (hd - a.Hq - a.Hkv) * a.D
                                  : k + t * a.ldk + (hd - a.Hq) * a.D);
        int64_t to = t;
        bool keep = in;
        if (!isq && slot != nullptr) {
            to = slot[t];
            keep = in && to >= 0 && to < a.n_slots;
        }
        E *dst = isq ? qo + t * a.ldqo + hd * a.D
                     : (isv ? vo + to * a.ldvo + (hd - a.Hq - a.Hkv) * a.D
                            : ko + to * a.ldko + (hd - a.Hq) * a.D);
        float x1[4] = {0, 0, 0, 0}, x2[4] = {0, 0, 0, 0};
        if (in) {
            load4(src + c, x1);
            load4(src + half + c, x2);
        }
        if (NORM) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                s = fmaf(x1[i], x1[i], fmaf(x2[i], x2[i], s));
            s = sum_lanes<L>(s);
            const float r = isv ? 1.f : 1.f / sqrtf(s / a.D + a.eps);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x1[i] *= r * (isv ? 1.f : isq ? wq1[i] : wk1[i]);
                x2[i] *= r * (isv ? 1.f : isq ? wq2[i] : wk2[i]);
            }
        }
        if (!keep)
            continue;
        if (!isv) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 w = cs[tt * half + c + i];
                const float y1 = x1[i], y2 = x2[i];
                x1[i] = fmaf(y1, w.x, -(y2 * w.y));
                x2[i] = fmaf(y2, w.x, y1 * w.y);
            }
        }
        save4(dst + c, x1);
        save4(dst + half + c, x2);
    }
}

// dx and, with the norm, the block's share of dw: [q, k][D] at
// part[blockIdx.x]
template <typename E, int L, bool NORM>
__global__ __launch_bounds__(256) void rotary_bwd_k(const E *q, const E *k, const E *wq,
                                                    const E *wk, const E *dqo, const E *dko, E *dq,
                                                    E *dk, float *part, RotaryArgs a, int per)
{
    __shared__ float2 cs[kTokens * 4 * L];
    __shared__ float red[NORM ? 256 * 9 : 1]; // 8 values a thread, one of padding
    const int half = a.D / 2;
    const int c = 4 * (threadIdx.x % L);
    const bool in = c < half;
    const int heads = a.Hq + a.Hkv;
    float w[2][8], dw[2][8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        w[0][i] = w[1][i] = 1.f, dw[0][i] = dw[1][i] = 0.f;
    if (NORM && in) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const E *p = s ? wk : wq;
            if (p != nullptr) {
                float u1[4], u2[4];
                load4(p + c, u1);
                load4(p + half + c, u2);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[s][i] = u1[i], w[s][4 + i] = u2[i];
            }
        }
    }
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * per; t0 < a.T;
         t0 += static_cast<int64_t>(gridDim.x) * per) {
        const int tokens = static_cast<int>(a.T - t0 < per ? a.T - t0 : per);
        __syncthreads();
        make_turns(cs, a, t0, tokens);
        __syncthreads();
        for (int e = threadIdx.x / L; e < tokens * heads; e += 256 / L) {
            const int tt = e / heads, hd = e - tt * heads;
            const int64_t t = t0 + tt;
            const bool isq = hd < a.Hq;
            const E *src = isq ? q + t * a.ldq + hd * a.D : k + t * a.ldk + (hd - a.Hq) * a.D;
            const E *grd = isq ? dqo + t * a.ldqo + hd * a.D : dko + t * a.ldko + (hd - a.Hq) * a.D;
            E *dst = isq ? dq + t * a.lddq + hd * a.D : dk + t * a.lddk + (hd - a.Hq) * a.D;
            float x[8] = {}, g[8] = {};
            if (in) {
                float u1[4], u2[4];
                if (NORM) {
                    load4(src + c, u1);
                    load4(src + half + c, u2);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        x[i] = u1[i], x[4 + i] = u2[i];
                }
                load4(grd + c, u1);
                load4(grd + half + c, u2);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 u = cs[tt * half + c + i];
                    g[i] = fmaf(u1[i], u.x, u2[i] * u.y);
                    g[4 + i] = fmaf(u2[i], u.x, -(u1[i] * u.y));
                }
            }
            if (NORM) {
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    s = fmaf(x[i], x[i], s);
                s = sum_lanes<L>(s);
                const float r = 1.f / sqrtf(s / a.D + a.eps);
                float dot = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] *= r;
                    const float d = g[i] * x[i];
                    dw[0][i] += isq ? d : 0.f;
                    dw[1][i] += isq ? 0.f : d;
                    g[i] *= isq ? w[0][i] : w[1][i];
                    dot = fmaf(g[i], x[i], dot);
                }
                dot = sum_lanes<L>(dot) / a.D;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    g[i] = r * fmaf(-x[i], dot, g[i]);
            }
            if (in) {
                float u1[4], u2[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    u1[i] = g[i], u2[i] = g[4 + i];
                save4(dst + c, u1);
                save4(dst + half + c, u2);
            }
        }
    }
    if (NORM) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i)
                red[threadIdx.x * 9 + i] = dw[s][i];
            __syncthreads();
            // element d: value d's place of the lanes that hold it
            for (int d = threadIdx.x; d < a.D; d += 256) {
                const int j = d < half ? d : d - half;
                const int lane = j / 4, at = j % 4 + (d < half ? 0 : 4);
                float v = 0.f;
                for (int i = 0; i < 256 / L; ++i)
                    v += red[(i * L + lane) * 9 + at];
                part[(static_cast<size_t>(blockIdx.x) * 2 + s) * a.D + d] = v;
            }
        }
    }
}

// dw[e] = sum over the blocks, 32 elements a block: 32 chains of them, added
// in order
__global__ __launch_bounds__(1024) void rotary_reduce_k(const float *part, int nparts, int D,
                                                        float *dwq, float *dwk)
{
    __shared__ float red[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int e = blockIdx.x * 32 + x;
    float v = 0.f;
    if (e < 2 * D)
#pragma unroll 8
        for (int i = y; i < nparts; i += 32)
            v += part[static_cast<size_t>(i) * 2 * D + e];
    red[y][x] = v;
    __syncthreads();
    if (y == 0 && e < 2 * D) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i)
            s += red[i][x];
        float *to = e < D ? dwq : dwk;
        if (to != nullptr)
            to[e < D ? e : e - D] = s;
    }
}

// kTokens tokens, fewer where that makes less than four blocks a compute unit
// (1000 tokens, 16 + 4 heads of 128 in bfloat16: forward 12.4 -> 6.2, backward
// 14.8 -> 8.0 us; 300 of 64 in float32: 6.3 -> 4.2, 8.5 -> 4.5); up to kTokens
// in all take one block (4 tokens: 4.5 us either way)
int tokens_per_block(int64_t T)
{
    int per = kTokens;
    while (T > kTokens && per > 1 && T / per < 4 * device_cus())
        per /= 2;
    return per;
}

template <typename E, int L>
hipError_t fwd(const void *q, const void *k, const void *v, const void *wq, const void *wk,
               void *qo, void *ko, void *vo, const int32_t *slot, const RotaryArgs &a,
               hipStream_t st)
{
    const int per = tokens_per_block(a.T);
    const dim3 grid(static_cast<uint32_t>((a.T + per - 1) / per));
    const auto p = [](const void *x) { return static_cast<const E *>(x); };
    const auto w = [](void *x) { return static_cast<E *>(x); };
    if (a.norm)
        HEX_LAUNCH((rotary_fwd_k<E, L, true>), grid, dim3(256), 0, st, p(q), p(k), p(v), p(wq),
                   p(wk), w(qo), w(ko), w(vo), slot, a, per);
    else
        HEX_LAUNCH((rotary_fwd_k<E, L, false>), grid, dim3(256), 0, st, p(q), p(k), p(v), p(wq),
                   p(wk), w(qo), w(ko), w(vo), slot, a, per);
    return hipGetLastError();
}

template <typename E, int L>
hipError_t bwd(const void *q, const void *k, const void *wq, const void *wk, const void *dqo,
               const void *dko, void *dq, void *dk, float *dwq, float *dwk, float *part,
               const RotaryArgs &a, hipStream_t st)
{
    const int blocks = rotary_bwd_blocks(a.T), per = tokens_per_block(a.T);
    const auto p = [](const void *x) { return static_cast<const E *>(x); };
    const auto w = [](void *x) { return static_cast<E *>(x); };
    if (!a.norm) {
        HEX_LAUNCH((rotary_bwd_k<E, L, false>), dim3(blocks), dim3(256), 0, st, p(q), p(k), p(wq),
                   p(wk), p(dqo), p(dko), w(dq), w(dk), part, a, per);
        return hipGetLastError();
    }
    HEX_LAUNCH((rotary_bwd_k<E, L, true>), dim3(blocks), dim3(256), 0, st, p(q), p(k), p(wq), p(wk),
               p(dqo), p(dko), w(dq), w(dk), part, a, per);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || (dwq == nullptr && dwk == nullptr))
        return e;
    HEX_LAUNCH(rotary_reduce_k, dim3((2 * a.D + 31) / 32), dim3(1024), 0, st, part, blocks, a.D,
               dwq, dwk);
    return hipGetLastError();
}

} // namespace

hipError_t rotary_zero(float *dwq, float *dwk, int D, hipStream_t st)
{
    if (dwq == nullptr && dwk == nullptr)
        return hipSuccess;
    HEX_LAUNCH(rotary_reduce_k, dim3((2 * D + 31) / 32), dim3(1024), 0, st, nullptr, 0, D, dwq,
               dwk);
    return hipGetLastError();
}

int rotary_bwd_blocks(int64_t T)
{
    const int per = tokens_per_block(T);
    const int64_t n = (T + per - 1) / per;
    const int64_t most = 4 * static_cast<int64_t>(device_cus());
    return static_cast<int>(n < most ? n : most);
}

hipError_t rotary_fwd(const void *q, const void *k, const void *v, const void *wq, const void *wk,
                      void *qo, void *ko, void *vo, const int32_t *slot, const RotaryArgs &a,
                      Dtype dt, hipStream_t st)
{
    const auto run = [&](auto f) { return f(q, k, v, wq, wk, qo, ko, vo, slot, a, st); };
    if (dt == F32)
        return a.D <= 32   ? run(fwd<float, 4>)
               : a.D <= 64 ? run(fwd<float, 8>)
                           : run(fwd<float, 16>);
    return a.D <= 32   ? run(fwd<bf16raw, 4>)
           : a.D <= 64 ? run(fwd<bf16raw, 8>)
                       : run(fwd<bf16raw, 16>);
}

hipError_t rotary_bwd(const void *q, const void *k, const void *wq, const void *wk,
                      const void *dqo, const void *dko, void *dq, void *dk, float *dwq, float *dwk,
                      float *part, const RotaryArgs &a, Dtype dt, hipStream_t st)
{
    const auto run = [&](auto f) {
        return f(q, k, wq, wk, dqo, dko, dq, dk, dwq, dwk, part, a, st);
    };
    if (dt == F32)
        return a.D <= 32   ? run(bwd<float, 4>)
               : a.D <= 64 ? run(bwd<float, 8>)
                           : run(bwd<float, 16>);
    return a.D <= 32   ? run(bwd<bf16raw, 4>)
           : a.D <= 64 ? run(bwd<bf16raw, 8>)
                       : run(bwd<bf16raw, 16>);
}

} // namespace hexk
