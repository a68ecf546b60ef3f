// k_pack.hip -- operands of the matrix product (gemm.h) from tensors that are
// not in its form, sums over rows, and zeros.  Bound by memory: 16432 x 512 of
// float32 into planes 17 us (5.0 TB/s), 51200 x 1024 of bfloat16 times act' 67 (4.7),
// their columns' sums 18 and 5 more.
#include "tokens.h"

namespace hexk {
namespace {

constexpr int kThreads = 256;

// One thread eight columns of a row of the destination: the source (or zeros
// past its rows and columns), times act'(z) where z is given, in one plane
// (bfloat16) or as the sum of three (float32).  A source of two halves of `half`
// rows puts the second at row `halfp`.
template <typename E> __global__ __launch_bounds__(kThreads) void pack_k(PackJobs jobs)
{
    int b = blockIdx.x, j = 0;
    while (j + 1 < jobs.n && b >= jobs.job[j].blocks) {
        b -= jobs.job[j].blocks;
        ++j;
    }
    const PackJob &q = jobs.job[j];
    // (fewer than 2^32 threads: check_linear and check_ffn)
    const uint32_t per = static_cast<uint32_t>(q.dld / 8);
    const uint32_t at = static_cast<uint32_t>(b) * kThreads + threadIdx.x, r = at / per;
    const int64_t row = r;
    if (row >= q.drows)
        return;
    const int col = static_cast<int>(at - r * per) * 8;
    int64_t from = row;
    bool in = row < q.rows;
    if (q.half > 0) {
        in = row < q.half || (row >= q.halfp && row < q.halfp + q.half);
        from = row < q.half ? row : row - q.halfp + q.half;
    }
    const int n = in ? q.cols - col : 0;
    const E *src = static_cast<const E *>(q.src) + (in ? from * q.ld + col : 0);
    float v[8];
    row8<E, false>(src, n, v);
    if (q.z != nullptr) {
        float z[8], a;
        row8<E, false>(static_cast<const E *>(q.z) + (in ? from * q.cols + col : 0), n, z);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] *= derivative<sizeof(E) == 4>(z[i], q.act, a);
        if (n < 8) // a derivative is not zero at the zeros behind a row
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = i < n ? v[i] : 0.f;
    }
    bf16raw *dst = q.dst + row * q.dld + col;
    if constexpr (sizeof(E) == 2)
        save_row8<bf16raw, true>(dst, 8, v);
    else
        save_planes(dst, q.plane, v);
}

// part[slice][column]: sums over a slice's rows of a matrix of E, or of three
// bfloat16 planes; a block takes 64 columns, 32 rows at a time
template <typename E>
__global__ __launch_bounds__(kThreads) void col_sum_k(const E *x, int64_t ld, int64_t plane,
                                                      int planes, int64_t rows, int cols, int vec,
                                                      int64_t slice, float *part)
{
    __shared__ float lds[32][65];
    const int g = threadIdx.x % 8, sub = threadIdx.x / 8, c = blockIdx.x * 64 + 8 * g;
    const int64_t r0 = blockIdx.y * slice, r1 = r0 + slice < rows ? r0 + slice : rows;
    float s[8] = {};
    if (c < cols)
        for (int64_t r = r0 + sub; r < r1; r += 32)
            for (int p = planes - 1; p >= 0; --p) {
                float v[8];
                if (vec)
                    row8<E, true>(x + p * plane + r * ld + c, cols - c, v);
                else
                    row8<E, false>(x + p * plane + r * ld + c, cols - c, v);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    s[i] += v[i];
            }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        lds[sub][8 * g + i] = s[i];
    __syncthreads();
    if (threadIdx.x >= 64 || blockIdx.x * 64 + threadIdx.x >= cols)
        return;
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k)
        t += lds[k][threadIdx.x];
    part[blockIdx.y * static_cast<int64_t>(cols) + blockIdx.x * 64 + threadIdx.x] = t;
}

constexpr int kJoin = 1024;
template <typename O>
__global__ __launch_bounds__(kJoin) void col_join_k(const float *part, int slices, int cols,
                                                    Halves map, O *out)
{
    __shared__ float lds[kJoin / 16][17];
    const int c = blockIdx.x * 16 + threadIdx.x % 16, sub = threadIdx.x / 16;
    float t = 0.f;
    if (c < cols)
#pragma unroll 8
        for (int s = sub; s < slices; s += kJoin / 16)
            t += part[static_cast<int64_t>(s) * cols + c];
    lds[sub][threadIdx.x % 16] = t;
    __syncthreads();
    const int to = c < cols ? map.row(c) : -1;
    if (sub != 0 || to < 0)
        return;
    t = 0.f;
#pragma unroll
    for (int s = 0; s < kJoin / 16; ++s)
        t += lds[s][threadIdx.x % 16];
    out[to] = from_f<O>(t);
}

// eight elements a thread, p 16-byte aligned: 2^33 elements, the most that check_linear
// and check_ffn let through, are 2^30 threads (a launch counts them in 32 bits)
template <typename O> __global__ __launch_bounds__(kThreads) void zero_k(O *p, int64_t n)
{
    const int64_t at = 8 * (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x);
    const float zeros[8] = {};
    if (at < n)
        save_row8<O, true>(p + at, n - at < 8 ? static_cast<int>(n - at) : 8, zeros);
}

} // namespace

hipError_t pack(PackJobs &jobs, Dtype dt, hipStream_t st)
{
    if (jobs.n == 0)
        return hipSuccess;
    int64_t blocks = 0;
    for (int j = 0; j < jobs.n; ++j) {
        PackJob &q = jobs.job[j];
        q.blocks = static_cast<int>((q.dld / 8 * q.drows + kThreads - 1) / kThreads);
        blocks += q.blocks;
    }
    const dim3 grid(static_cast<uint32_t>(blocks));
    if (dt == F32)
        HEX_LAUNCH((pack_k<float>), grid, dim3(kThreads), 0, st, jobs);
    else
        HEX_LAUNCH((pack_k<bf16raw>), grid, dim3(kThreads), 0, st, jobs);
    return hipGetLastError();
}

int col_sum_slices(int64_t rows, int cols)
{
    // four blocks a compute unit, each at least 64 rows
    const int64_t across = (cols + 63) / 64;
    int64_t n = 4 * static_cast<int64_t>(device_cus()) / across;
    const int64_t most = (rows + 63) / 64;
    n = n > most ? most : n;
    return static_cast<int>(n < 1 ? 1 : n > 1024 ? 1024 : n);
}

hipError_t col_sum(const void *x, int64_t ld, int64_t plane, int planes, int64_t rows, int cols,
                   Halves map, float *part, void *out, Dtype src, Dtype dst, hipStream_t st)
{
    const int slices = col_sum_slices(rows, cols);
    const int64_t slice = (rows + slices - 1) / slices;
    const dim3 grid(static_cast<uint32_t>((cols + 63) / 64), static_cast<uint32_t>(slices));
    const int vec = ld % (src == F32 ? 4 : 8) == 0 && plane % 8 == 0;
    if (src == F32)
        HEX_LAUNCH((col_sum_k<float>), grid, dim3(kThreads), 0, st, static_cast<const float *>(x),
                   ld, plane, planes, rows, cols, vec, slice, part);
    else
        HEX_LAUNCH((col_sum_k<bf16raw>), grid, dim3(kThreads), 0, st,
                   static_cast<const bf16raw *>(x), ld, plane, planes, rows, cols, vec, slice, part);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    const dim3 join(static_cast<uint32_t>((cols + 15) / 16));
    if (dst == F32)
        HEX_LAUNCH((col_join_k<float>), join, dim3(kJoin), 0, st, part, slices, cols, map,
                   static_cast<float *>(out));
    else
        HEX_LAUNCH((col_join_k<bf16raw>), join, dim3(kJoin), 0, st, part, slices, cols, map,
                   static_cast<bf16raw *>(out));
    return hipGetLastError();
}

hipError_t zero_fill(void *p, int64_t n, Dtype dt, hipStream_t st)
{
    if (p == nullptr || n == 0)
        return hipSuccess;
    const int64_t per = 8 * kThreads;
    const dim3 grid(static_cast<uint32_t>((n + per - 1) / per));
    if (dt == F32)
        HEX_LAUNCH((zero_k<float>), grid, dim3(kThreads), 0, st, static_cast<float *>(p), n);
    else
        HEX_LAUNCH((zero_k<bf16raw>), grid, dim3(kThreads), 0, st, static_cast<bf16raw *>(p), n);
    return hipGetLastError();
}

} // namespace hexk
