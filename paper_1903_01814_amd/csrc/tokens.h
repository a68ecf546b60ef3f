// tokens.h -- what the projections and the feed-forward block share beside the
// matrix product: operands laid out for it, sums over rows, workspaces.
#pragma once

#include "act.h"
#include "attn.h"
#include "gemm_plan.h"

namespace hexk {

// f<E, ACT>(args) for the type `dt` and the activation `act`
#define HEX_BY_ACT(f, E, ...)                                                                 \
    (act == ACT_RELU   ? f<E, ACT_RELU>(__VA_ARGS__)                                          \
     : act == ACT_GELU ? f<E, ACT_GELU>(__VA_ARGS__)                                          \
     : act == ACT_SILU ? f<E, ACT_SILU>(__VA_ARGS__)                                          \
                       : f<E, ACT_NONE>(__VA_ARGS__))
#define HEX_BY_TYPE(f, ...)                                                                   \
    (dt == F32 ? HEX_BY_ACT(f, float, __VA_ARGS__) : HEX_BY_ACT(f, bf16raw, __VA_ARGS__))

constexpr int64_t round8(int64_t n) { return (n + 7) / 8 * 8; }
// Columns of a row that the library lays out: whole vectors, and past 256 columns whole
// cache lines, as a row's part of a tile would lie in two lines else (bfloat16, 16384
// tokens, 5464 to 2048 features: 358 us, with x's rows 5504 apart 348, with 5504
// features, so that w's are too, 314; weights' gradient 386 and with x's rows 5504
// apart 366; weights' gradient of rows of 10928 and of 10944 705 and 678, data gradient
// 629 and 571).
constexpr int64_t pitch(int64_t n) { return n <= 256 ? round8(n) : (n + 63) / 64 * 64; }

// Two halves of `half` rows (or columns), the second from `halfp` on, as one run
// without the rows between; none (half = 0): as they are.
struct Halves {
    int half, halfp;
    __host__ __device__ __forceinline__ int row(int r) const
    {
        if (half == 0 || r < half)
            return r;
        return r >= halfp && r < halfp + half ? r - halfp + half : -1;
    }
};

// A tensor [rows][cols], rows `ld` apart, to dst [planes][drows][dld], zeros
// behind rows and columns; with z (dense) times act'(z).  half, halfp: the source
// has two halves (Halves), the second goes to row halfp.
struct PackJob {
    const void *src, *z;
    bf16raw *dst;
    int64_t ld, dld, plane, drows;
    int rows, cols, half, halfp, act;
    int blocks; // set by the launcher
};
struct PackJobs {
    PackJob job[4];
    int n;
};
hipError_t pack(PackJobs &jobs, Dtype dt, hipStream_t st);

// out[map(c)] = sum over the rows of column c; part: col_sum_slices(rows, cols) *
// cols floats.  x: float32 or bfloat16, or three bfloat16 planes.
int col_sum_slices(int64_t rows, int cols);
hipError_t col_sum(const void *x, int64_t ld, int64_t plane, int planes, int64_t rows, int cols,
                   Halves map, float *part, void *out, Dtype src, Dtype dst, hipStream_t st);

// v as three bfloat16 numbers each (attn.h, Split), in planes `plane` elements
// apart
__device__ __forceinline__ void save_planes(bf16raw *dst, int64_t plane, float (&v)[8])
{
    const attn::FragSplit f = attn::split8(v);
#pragma unroll
    for (int p = 0; p < 3; ++p)
        *reinterpret_cast<uint4 *>(dst + p * plane) = __builtin_bit_cast(uint4, f.p[p]);
}

// A workspace handed out in pieces of whole 256 bytes; without memory behind it
// it only counts.
struct Space {
    char *base;
    size_t used = 0;
    template <typename T> T *take(int64_t n)
    {
        T *p = base == nullptr ? nullptr : reinterpret_cast<T *>(base + used);
        used += (static_cast<size_t>(n) * sizeof(T) + 255) / 256 * 256;
        return p;
    }
};

namespace gemm {
struct Side;
}
// The product's operand of a tensor [rows][cols]: itself, or (float32, rows of
// parts of vectors, two halves that are, an activation's gradient) a place in the
// workspace and the job that fills it.  copy: a place in any case, for rows that begin
// on cache lines.
gemm::Side operand(const void *src, const void *z, int act, int rows, int cols, int64_t ld, Dtype dt,
                   Halves map, Space &ws, PackJobs &jobs, bool copy = false);
// its columns as the operand's rows
gemm::Side tall(const gemm::Side &s, int cols);

// What a projection's sums become: y = act(z) + res, z = sums + bias.
struct Output {
    const void *bias, *res;
    void *y, *z;
    int64_t ldr, ldy;
};
// of operands W and X
hipError_t linear_product(const gemm::Plan &pl, const gemm::Side &W, const gemm::Side &X, float *ws,
                          const Output &o, int act, Dtype dt, hipStream_t st);
// of a few tokens, tensors as they are
hipError_t linear_few(const void *w, const void *x, int64_t ldx, int M, int N, int K,
                      const Output &o, int act, Dtype dt, hipStream_t st);
// y [map(m)] = Q P in dt: P tall, Q wide (data gradient) or tall (weight gradient);
// sums[map(m)], where not null (Q tall, gemm::gives_sums), the sums of Q over k
hipError_t store_product(bool tall_q, const gemm::Plan &pl, const gemm::Side &P,
                         const gemm::Side &Q, float *ws, void *y, int64_t ldy, void *sums,
                         Halves map, Dtype dt, hipStream_t st);

} // namespace hexk
