// act.h -- activations and their derivatives, and rows of eight elements, as
// the token-wise kernels (norm, linear, feed-forward) share them.
#pragma once

#include <type_traits>

#include "hexdev.h"
#include "kernels.h"

namespace hexk {

// 1 / (1 + exp(-z)).  float32 calls take the library's exponential; bfloat16
// ones the hardware's, whose error (the rounding of z log2(e), 2^-24 |z|) is far
// below the result's rounding.
template <bool FINE> __device__ __forceinline__ float sigmoid(float z)
{
    if constexpr (FINE)
        return 1.f / (1.f + expf(-z));
    else
        return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
}

// The normal distribution's function (1 + erf(z / sqrt 2)) / 2.  bfloat16: Abramowitz
// and Stegun 7.1.26, erf(x) = 1 - (a1 t + .. + a5 t^5) exp(-x^2) with t = 1 / (1
// + p x), off by 1.5e-7 at most, so that its tail keeps bfloat16's bits down to
// 4e-5 (z = -4); a gelu output z phi is off by 6e-7 there, 2^-20.  In the epilogue of
// 51200 x 1024 x 1024 it takes 11 of 141 us.
template <bool FINE> __device__ __forceinline__ float normal_cdf(float z)
{
    if constexpr (FINE) {
        return 0.5f * erfcf(-0.70710678118654752f * z);
    } else {
        const float x = fabsf(z) * 0.70710678118654752f;
        const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
        float p = fmaf(1.061405429f, t, -1.453152027f);
        p = fmaf(p, t, 1.421413741f);
        p = fmaf(p, t, -0.284496736f);
        p = fmaf(p, t, 0.254829592f);
        // half of the upper tail
        const float q = 0.5f * p * t * __builtin_amdgcn_exp2f(-1.4426950408889634f * x * x);
        return z < 0.f ? q : 1.f - q;
    }
}

// act(z).  An infinity gives the limit (0 at minus infinity), a NaN a NaN.
template <bool FINE> __device__ __forceinline__ float activate(float z, int act)
{
    switch (act) {
    case ACT_RELU:
        return z < 0.f ? 0.f : z; // NaN stays
    case ACT_GELU: {
        const float p = normal_cdf<FINE>(z);
        return p == 0.f ? 0.f : z * p;
    }
    case ACT_SILU: {
        const float s = sigmoid<FINE>(z);
        return s == 0.f ? 0.f : z * s;
    }
    default:
        return z;
    }
}

// act(z) and act'(z)
template <bool FINE> __device__ __forceinline__ float derivative(float z, int act, float &a)
{
    switch (act) {
    case ACT_RELU:
        a = z < 0.f ? 0.f : z;
        return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    case ACT_GELU: {
        const float p = normal_cdf<FINE>(z);
        a = p == 0.f ? 0.f : z * p;
        float e;
        if constexpr (FINE)
            e = expf(-0.5f * z * z);
        else
            e = __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
        return e == 0.f ? p : fmaf(z * e, 0.39894228040143268f, p);
    }
    case ACT_SILU: {
        const float s = sigmoid<FINE>(z);
        a = s == 0.f ? 0.f : z * s;
        return s == 0.f || s == 1.f ? s : s * fmaf(z, 1.f - s, 1.f);
    }
    default:
        a = z;
        return 1.f;
    }
}

// Eight elements of a row from p on, the first n of them (zeros behind); one
// load each 16 bytes where all are there, at any alignment of the element's size
// unless the address is known to be a multiple of 16 (VEC).
template <typename E> __device__ __forceinline__ void unpack8(const uint4 *u, float (&v)[8])
{
    if constexpr (sizeof(E) == 2) {
        const uint32_t w[4] = {u[0].x, u[0].y, u[0].z, u[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v[4 * i] = __uint_as_float(u[i].x), v[4 * i + 1] = __uint_as_float(u[i].y);
            v[4 * i + 2] = __uint_as_float(u[i].z), v[4 * i + 3] = __uint_as_float(u[i].w);
        }
    }
}
template <typename E> __device__ __forceinline__ void pack8(const float (&v)[8], uint4 *u)
{
    if constexpr (sizeof(E) == 2) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = from_f<bf16raw>(v[2 * i]) |
                   static_cast<uint32_t>(from_f<bf16raw>(v[2 * i + 1])) << 16;
        u[0] = uint4{w[0], w[1], w[2], w[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            u[i] = uint4{__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                         __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
    }
}
// the elements as they lie in memory, to be unpacked later
template <typename E> struct Raw8 {
    uint4 u[sizeof(E) / 2];
};
template <typename E, bool VEC> __device__ __forceinline__ Raw8<E> raw8(const E *p, int n)
{
    Raw8<E> r = {};
    if (n >= 8) {
        if constexpr (VEC) {
#pragma unroll
            for (int q = 0; q < static_cast<int>(sizeof(E) / 2); ++q)
                r.u[q] = reinterpret_cast<const uint4 *>(p)[q];
        } else {
            __builtin_memcpy(r.u, p, sizeof(r.u)); // at any element
        }
    } else if (n > 0) {
        E v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = i < n ? p[i] : E(0);
        __builtin_memcpy(r.u, v, sizeof(v));
    }
    return r;
}
template <typename E, bool VEC>
__device__ __forceinline__ void row8(const E *p, int n, float (&v)[8])
{
    unpack8<E>(raw8<E, VEC>(p, n).u, v);
}
template <typename E, bool VEC>
__device__ __forceinline__ void save_row8(E *p, int n, const float (&v)[8])
{
    constexpr int Q = sizeof(E) / 2;
    if (n >= 8) {
        uint4 u[Q];
        pack8<E>(v, u);
        if constexpr (VEC) {
#pragma unroll
            for (int q = 0; q < Q; ++q)
                reinterpret_cast<uint4 *>(p)[q] = u[q];
        } else {
            __builtin_memcpy(p, u, sizeof(u));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n)
                p[i] = from_f<E>(v[i]);
    }
}

} // namespace hexk
