// attn.h -- what the attention kernels share: matrix-core operands of either
// type, the LDS layout of a staged tile, where blocks run.  Which rows of which
// sequence a block takes is in attn_span.h.
//
// All products are 32 x 32 (x 16 in bfloat16, x 2 in float32).  An operand
// ("fragment") is 8 contraction elements of one row per lane: row = lane % 32,
// half h = lane / 32.  Result register r of a lane holds row
// (r % 4) + 8 (r / 4) + 4 h of column lane % 32.
//
// The scores are computed with the sequence axis that is contracted next as
// the result's rows.  A lane's registers 8 s .. 8 s + 7 are then, without any
// exchange between lanes, the operand of the next product, whose contraction
// index is the row 16 s + 8 (i / 4) + 4 h + i % 4 for element i; the other
// operand is read from LDS with rows in the same order (read_rows).
#pragma once

#include "attn_span.h"
#include "hexdev.h"
#include "kernels.h"

namespace hexk {
namespace attn {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

// log2(e) and ln(2) as a float and what it leaves
constexpr float kLog2e = 1.4426950408889634f, kLog2eLo = 1.4426950408889634 - kLog2e;
constexpr float kLn2 = 0.6931471805599453f, kLn2Lo = 0.6931471805599453 - kLn2;

// ---- how a type is multiplied.  E: what tensors hold; Frag: an operand;
// Score: a sum over the head dimension while it is added up; FINE: exponents
// in two parts (prob).  In LDS an element takes BYTES bytes in each of PLANES
// tiles.
//
// bfloat16: as it is.
struct Bf16 {
    using E = bf16raw;
    using Frag = bf16x8;
    using Score = floatx16;
    static constexpr bool FINE = false;
    static constexpr int BYTES = 2, PLANES = 1;
};
// float32 as three bfloat16 numbers, x = h + m + l: h is x rounded, m the rest
// rounded, l the rest of that, 8 bits each, so that nothing is left out of the
// 24.  A product is the six products h h', h m', m h', m m', h l', l h' in
// float32 sums; what is dropped is 2^-24 of it, a rounding of a float32
// product.  Six bfloat16 products take 192 clocks where the float32 ones take
// 512 (32 x 32 x 16); the kernels gain 1.4 to 1.8 (D = 32 to 128).  Values
// below 2^-110 lose bits (their rests are denormal); infinities, and finite
// values from 3.39e38 on, which round to one, become NaN.
struct FragSplit {
    bf16x8 p[3];
};
struct ScoreSplit {
    floatx16 hi, lo; // h h', and the rest
};
struct Split {
    using E = float;
    using Frag = FragSplit;
    using Score = ScoreSplit;
    static constexpr bool FINE = true;
    static constexpr int BYTES = 2, PLANES = 3;
};
// float32 as it is, for the cache step: each of its waves has tiles of its own,
// whose three parts do not fit LDS, and it waits for memory either way.
struct FragF32 {
    float v[8];
};
struct Full {
    using E = float;
    using Frag = FragF32;
    using Score = floatx16;
    static constexpr bool FINE = true;
    static constexpr int BYTES = 4, PLANES = 1;
};

// Whole sequences of E are multiplied by Math<E>, with so many waves a SIMD:
// two, while the operands fit 256 registers.
template <typename E> using Math = std::conditional_t<sizeof(E) == 2, Bf16, Split>;
constexpr int attn_waves(bool f32, int DC) { return f32 && DC > 64 ? 1 : 2; }

__device__ __forceinline__ floatx16 mma(bf16x8 a, bf16x8 b, floatx16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// the five small products of two split operands, then the large one
__device__ __forceinline__ floatx16 mma_rest(const FragSplit &a, const FragSplit &b, floatx16 c)
{
    c = mma(a.p[2], b.p[0], c);
    c = mma(a.p[0], b.p[2], c);
    c = mma(a.p[1], b.p[1], c);
    c = mma(a.p[1], b.p[0], c);
    return mma(a.p[0], b.p[1], c);
}
__device__ __forceinline__ floatx16 mma(const FragSplit &a, const FragSplit &b, floatx16 c)
{
    return mma(a.p[0], b.p[0], mma_rest(a, b, c));
}
__device__ __forceinline__ floatx16 mma(const FragF32 &a, const FragF32 &b, floatx16 c)
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[i], b.v[i], c, 0, 0, 0);
    return c;
}

// The next 16 elements of a score.  Scores of 100, whose exponentials carry
// 100 times their relative error, are where float32's roundings count: so Full
// adds 16 elements at a time from zero and these sums by the vector unit (8
// roundings of the score's size at D = 128, not 64), and Split keeps its large
// products apart from the small ones.
__device__ __forceinline__ void add_product(bf16x8 a, bf16x8 b, floatx16 &c) { c = mma(a, b, c); }
__device__ __forceinline__ void add_product(const FragF32 &a, const FragF32 &b, floatx16 &c)
{
    c = c + mma(a, b, floatx16{});
}
__device__ __forceinline__ void add_product(const FragSplit &a, const FragSplit &b, ScoreSplit &c)
{
    c.lo = mma_rest(a, b, c.lo);
    c.hi = mma(a.p[0], b.p[0], c.hi);
}
__device__ __forceinline__ floatx16 value(const floatx16 &c) { return c; }
__device__ __forceinline__ floatx16 value(const ScoreSplit &c) { return c.hi + c.lo; }

__device__ __forceinline__ bf16x8 round8(const float (&v)[8])
{
    bf16x8 f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        f[i] = static_cast<__bf16>(v[i]);
    return f;
}
__device__ __forceinline__ FragSplit split8(float (&v)[8])
{
    FragSplit f;
#pragma unroll
    for (int p = 0; p < 3; ++p) {
        f.p[p] = round8(v);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] -= static_cast<float>(f.p[p][i]);
    }
    return f;
}
template <typename M> __device__ __forceinline__ typename M::Frag make_frag(float (&v)[8])
{
    if constexpr (M::PLANES == 3) {
        return split8(v);
    } else if constexpr (M::BYTES == 2) {
        return round8(v);
    } else {
        FragF32 f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f.v[i] = v[i];
        return f;
    }
}

// A number of powers of two as hi + lo, and 2^(x scale log2(e) - ref).  At
// scores of 100 the rounding of the factor and of the reference alone would
// put float32 probabilities off by 1e-5; so there both are kept in two parts.
struct Ref {
    float hi, lo;
};
__device__ __forceinline__ Ref ref_of_lse(float lse)
{
    const float hi = lse * kLog2e;
    return Ref{hi, fmaf(lse, kLog2eLo, fmaf(lse, kLog2e, -hi))};
}
template <typename M>
__device__ __forceinline__ float prob(float x, const AttnArgs &a, float hi, float lo)
{
    float e = fmaf(x, a.c, -hi);
    if constexpr (M::FINE)
        e += fmaf(x, a.c_lo, -lo);
    return __builtin_amdgcn_exp2f(e);
}
// log of a sum l of 2^(.. - m), in units of e, with one rounding of its size
__device__ __forceinline__ float log_sum(float m, float l)
{
    return fmaf(m, kLn2, fmaf(m, kLn2Lo, __builtin_amdgcn_logf(l) * kLn2));
}

// Registers 8 s .. 8 s + 7 of a result as an operand; bfloat16 rounds to
// nearest even (probabilities lie in [0, 1], their sum is kept in float32
// from the unrounded values).
template <typename M> __device__ __forceinline__ typename M::Frag to_frag(const floatx16 &x, int s)
{
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = x[8 * s + i];
    return make_frag<M>(v);
}

// ---- tiles in LDS: rows of DC head elements (a multiple of 32, padded with
// zeros), 16-byte chunks permuted within the row by its number, so that both
// reads below spread over all 64 banks: sixteen rows of one chunk
// (read_cols), and runs of 64 or 128 bytes of four to eight rows (read_rows).
template <typename M, int DC, int ROWS> struct Tile {
    using Frag = typename M::Frag;
    static constexpr int PITCH = (DC == 96 ? 128 : DC) * M::BYTES; // bytes a row
    static constexpr int PLANE = ROWS * PITCH, SIZE = M::PLANES * PLANE;

    __device__ __forceinline__ static int swz(int row)
    {
        if constexpr (M::BYTES == 2) {
            if constexpr (PITCH == 256)
                return ((row >> 2) & 3) | (row & 3) << 2;
            else if constexpr (PITCH == 128)
                return ((row >> 2) & 3) | (row & 2) << 1;
            else
                return (row >> 2) & 3;
        } else {
            if constexpr (PITCH >= 256)
                return (row & 3) | (row & 4) << 1 | (row & 8) >> 1;
            else
                return (row >> 1) & 7;
        }
    }
    __device__ __forceinline__ static int chunk_at(int row, int chunk)
    {
        return row * PITCH + ((chunk ^ swz(row)) << 4);
    }

    // Operand with the head dimension as contraction: row `row` (per lane),
    // elements 16 s + 8 h ..  The lane's part of its address is made once
    // (cols_at), a step changes it by an exclusive or, rows by an offset.
    __device__ __forceinline__ static int cols_at(int row, int h)
    {
        return row * PITCH + (((M::BYTES == 2 ? h : 2 * h) ^ swz(row)) << 4);
    }
    __device__ __forceinline__ static Frag read_cols(const unsigned char *t, int at, int s)
    {
        Frag f;
        if constexpr (M::PLANES == 3) {
#pragma unroll
            for (int p = 0; p < 3; ++p)
                f.p[p] = *reinterpret_cast<const bf16x8 *>(t + p * PLANE + (at ^ (s << 5)));
        } else if constexpr (M::BYTES == 2) {
            f = *reinterpret_cast<const bf16x8 *>(t + (at ^ (s << 5)));
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 u = *reinterpret_cast<const float4 *>(t + (at ^ (s << 6 | j << 4)));
                f.v[4 * j] = u.x, f.v[4 * j + 1] = u.y, f.v[4 * j + 2] = u.z, f.v[4 * j + 3] = u.w;
            }
        }
        return f;
    }

    // Operand with rows as contraction, in the order of a result's registers:
    // element i is row row0 + 8 (i / 4) + 4 h + i % 4 (row0 a multiple of 16),
    // column 32 d + lane % 32.  bfloat16: the transposing read (16 lanes read
    // four rows of 16 columns, lane i of them receives column i of the four
    // rows).
    struct RowsAt {
        int a, b;
    };
    __device__ __forceinline__ static RowsAt rows_at(int lane)
    {
        const int h = lane >> 5;
        if constexpr (M::BYTES == 2) {
            const int r = 4 * h + ((lane & 15) >> 2);
            const int c = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), o = 8 * (lane & 1);
            return RowsAt{chunk_at(r, c) + o, chunk_at(r + 8, c) + o};
        } else {
            return RowsAt{chunk_at(4 * h, (lane & 31) >> 2) + 4 * (lane & 3), 0};
        }
    }
    __device__ __forceinline__ static bf16x8 transposed(unsigned char *t, RowsAt at, int d)
    {
        using lp = __attribute__((address_space(3))) shortx4 *;
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(t + (at.a ^ (d << 6))));
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(t + (at.b ^ (d << 6))));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    __device__ __forceinline__ static Frag read_rows(unsigned char *t, RowsAt at, int row0, int d)
    {
        if constexpr (M::PLANES == 3) {
            Frag f;
#pragma unroll
            for (int p = 0; p < 3; ++p)
                f.p[p] = transposed(t + p * PLANE + row0 * PITCH, at, d);
            return f;
        } else if constexpr (M::BYTES == 2) {
            return transposed(t + row0 * PITCH, at, d);
        } else {
            // the permutation of row 8 (i / 4) + 4 h + i % 4 is that of row 4 h
            // and that of the rest, by exclusive or
            Frag f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = 8 * (i >> 2) + (i & 3);
                f.v[i] = *reinterpret_cast<const float *>(t + (row0 + r) * PITCH +
                                                          (at.a ^ (d << 7 | swz(r) << 4)));
            }
            return f;
        }
    }
};

// Keeps the compiler from making all of a loop's LDS addresses before the loop
// and holding them in registers: they cost one exclusive or each.
__device__ __forceinline__ void in_loop(int &v) { asm volatile("" : "+v"(v)); }

// the sum, and the maximum, of a lane's value and lane ^ 32's: the swap gives
// both lanes the lower half's value and the upper half's
struct Halves {
    float lower, upper;
};
__device__ __forceinline__ Halves halves(float v)
{
    const int i = __builtin_bit_cast(int, v);
    const auto r = __builtin_amdgcn_permlane32_swap(i, i, false, false);
    const uint32_t a = r[0], b = r[1]; // a bit cast of r[1] itself reads r[0]
    return Halves{__uint_as_float(a), __uint_as_float(b)};
}
__device__ __forceinline__ float both_sum(float v)
{
    const Halves x = halves(v);
    return x.lower + x.upper;
}
__device__ __forceinline__ float both_max(float v)
{
    const Halves x = halves(v);
    return fmaxf(x.lower, x.upper);
}

// 8 head elements of a row from global memory, zeros past D; `p` is the row's
// start (16-byte aligned), c the first element (a multiple of 8, as D).
__device__ __forceinline__ void load8(const float *p, int c, int D, float (&v)[8])
{
    float4 u{0, 0, 0, 0}, w{0, 0, 0, 0};
    if (c < D) {
        u = *reinterpret_cast<const float4 *>(p + c);
        w = *reinterpret_cast<const float4 *>(p + c + 4);
    }
    v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
    v[4] = w.x, v[5] = w.y, v[6] = w.z, v[7] = w.w;
}
__device__ __forceinline__ bf16x8 load8(const bf16raw *p, int c, int D)
{
    uint4 u{0, 0, 0, 0};
    if (c < D)
        u = *reinterpret_cast<const uint4 *>(p + c);
    return __builtin_bit_cast(bf16x8, u);
}
// the same as an operand
template <typename M>
__device__ __forceinline__ typename M::Frag load_frag(const typename M::E *p, int c, int D)
{
    if constexpr (sizeof(typename M::E) == 2) {
        return load8(p, c, D);
    } else {
        float v[8];
        load8(p, c, D, v);
        return make_frag<M>(v);
    }
}
__device__ __forceinline__ float dot8(const float *a, const float *b, int c, int D, float s)
{
    float x[8], y[8];
    load8(a, c, D, x);
    load8(b, c, D, y);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        s = fmaf(x[i], y[i], s);
    return s;
}
__device__ __forceinline__ float dot8(const bf16raw *a, const bf16raw *b, int c, int D, float s)
{
    const bf16x8 x = load8(a, c, D), y = load8(b, c, D);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        s = fmaf(static_cast<float>(x[i]), static_cast<float>(y[i]), s);
    return s;
}

// ---- packed sequences ----------------------------------------------------
// Sequences of so few rows on average take tiles of 64 rows and 32 keys, which
// they fill better, instead of 128 and 64 (forward, dq; 8 heads of 32, 512
// sequences of 130 rows: 69.8 -> 63.4, 84.0 -> 76.5 us; 4 of 64, 384 of 195:
// 54.2 -> 51.3, 71.9 -> 68.5; 256 of 345: 74.7 -> 75.3, 96.8 -> 94.3).  Not in
// float32, where every wave more splits the same keys again (4 heads of 64, 384
// of 95 rows: 52 -> 67, 81 -> 91).
constexpr int kShortRows = 256;
inline bool attn_short(const AttnArgs &a)
{
    return static_cast<int64_t>(a.Tq) * a.group.G < static_cast<int64_t>(kShortRows) * a.S;
}
// blocks of a launch over all slots and key heads
inline uint32_t attn_blocks(const AttnArgs &a)
{
    return static_cast<uint32_t>(a.narrow ? (a.slots + 7) / 8 * 8 : a.slots) * a.Hkv;
}

// keys of sequence s: its k_len from k_start on, or up to the next start; its
// queries' own tokens (q0, nq) where both have the same offsets
__device__ __forceinline__ void key_span(const AttnArgs &a, int s, int q0, int nq, int &begin,
                                         int &n)
{
    if (a.k_start == a.q_start && a.k_len == nullptr && a.Tk == a.Tq) {
        begin = q0;
        n = nq;
        return;
    }
    begin = min(max(a.k_start[s], 0), a.Tk);
    const int end = a.k_len != nullptr ? a.k_len[s] : a.k_start[s + 1] - begin;
    n = min(min(max(end, 0), a.max_len), a.Tk - begin);
}

// four results in a row of an output (8- or 16-byte aligned)
__device__ __forceinline__ void store4(float *p, float x, float y, float z, float w)
{
    *reinterpret_cast<float4 *>(p) = float4{x, y, z, w};
}
__device__ __forceinline__ void store4(bf16raw *p, float x, float y, float z, float w)
{
    *reinterpret_cast<ushort4 *>(p) =
        ushort4{from_f<bf16raw>(x), from_f<bf16raw>(y), from_f<bf16raw>(z), from_f<bf16raw>(w)};
}

// registers 4 i .. 4 i + 3
__device__ __forceinline__ float4 quad(const floatx16 &x, int i)
{
    return float4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
}
__device__ __forceinline__ void set_quad(floatx16 &x, int i, const float4 &y)
{
    x[4 * i] = y.x, x[4 * i + 1] = y.y, x[4 * i + 2] = y.z, x[4 * i + 3] = y.w;
}
__device__ __forceinline__ void add_quad(floatx16 &x, int i, const float4 &y)
{
    x[4 * i] += y.x, x[4 * i + 1] += y.y, x[4 * i + 2] += y.z, x[4 * i + 3] += y.w;
}

// one lane's results of a column: registers 4 i .. 4 i + 3 are elements
// c0 + 8 i .. of the row at p, those below D are stored, times f
template <typename E>
__device__ __forceinline__ void store_col(E *p, const floatx16 &x, int c0, int D, float f)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (c0 + 8 * i < D)
            store4(p + c0 + 8 * i, x[4 * i] * f, x[4 * i + 1] * f, x[4 * i + 2] * f,
                   x[4 * i + 3] * f);
}

// One tile on its way from memory to LDS: ROWS rows, a 16-byte chunk a thread
// at a time, NT threads.  Addresses are a uniform base and a 32-bit offset
// (token strides are below 2^24 bytes), so that a load costs two or three
// vector instructions beside itself.  Chunks past D stay zero.
template <typename M, int DC, int ROWS, int NT> struct Stage {
    using E = typename M::E;
    using TL = Tile<M, DC, ROWS>;
    // an item: what fills one 16-byte chunk of each plane
    static constexpr int ELEMS = 16 / M::BYTES, VECS = ELEMS * static_cast<int>(sizeof(E)) / 16;
    static constexpr int PER_ROW = DC / ELEMS, ITEMS = ROWS * PER_ROW, N = (ITEMS + NT - 1) / NT;
    uint4 r[N][VECS];

    __device__ __forceinline__ Stage()
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < VECS; ++j)
                r[i][j] = uint4{0, 0, 0, 0};
    }
    __device__ __forceinline__ static int row(int i)
    {
        return (threadIdx.x % NT + NT * i) / PER_ROW;
    }
    __device__ __forceinline__ static int item(int i)
    {
        return (threadIdx.x % NT + NT * i) % PER_ROW;
    }
    // (a thread's last may be past the tile's end)
    __device__ __forceinline__ static bool has(int i)
    {
        return (i + 1) * NT <= ITEMS || threadIdx.x % NT + NT * i < ITEMS;
    }
    // the item's place in its row, in bytes
    __device__ __forceinline__ static uint32_t place(int i) { return 16 * VECS * item(i); }
    __device__ __forceinline__ void get(int i, const E *base, uint32_t bytes, int D)
    {
        if (has(i) && item(i) * ELEMS < D)
#pragma unroll
            for (int j = 0; j < VECS; ++j)
                r[i][j] = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(base) +
                                                          bytes)[j];
    }
    // rows from `base` on, ld bytes apart; those past the last of `left`
    // repeat it
    __device__ __forceinline__ void rows(const E *base, uint32_t ld, int left, int D)
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
            get(i, base, __umul24(min(row(i), left - 1), ld) + place(i), D);
    }
    __device__ __forceinline__ void put(unsigned char *t) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (!has(i))
                break;
            unsigned char *to = t + TL::chunk_at(row(i), item(i));
            if constexpr (M::PLANES == 3) {
                float v[8] = {__uint_as_float(r[i][0].x), __uint_as_float(r[i][0].y),
                              __uint_as_float(r[i][0].z), __uint_as_float(r[i][0].w),
                              __uint_as_float(r[i][1].x), __uint_as_float(r[i][1].y),
                              __uint_as_float(r[i][1].z), __uint_as_float(r[i][1].w)};
                const FragSplit f = split8(v);
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    *reinterpret_cast<bf16x8 *>(to + p * TL::PLANE) = f.p[p];
            } else {
                *reinterpret_cast<uint4 *>(to) = r[i][0];
            }
        }
    }
};

// Which (key head, tile slot) block `id` takes.  Dies take blocks in turn, 8 of
// them.  Usually key heads are innermost, so that a head's keys stay on few
// dies.  Heads of less than a 128-byte cache line share lines with their
// neighbours: there all heads of a slot go to one die (512 sequences of 20 to
// 400 tokens, 8 heads of 32 in bfloat16: dq 81.4 -> 76.5 us, forward the same).
// Neighbouring slots go to different dies in either form, so the keys of a
// sequence are fetched once for each of its tiles, up to eight times (that
// batch: 3.8 times, forward 296 MB read where 100 would do).
// Slots from the last on: under the causal mask a sequence's last tiles are the
// longest.
__device__ __forceinline__ void head_and_slot(const AttnArgs &a, uint32_t id, int &kvh, int &slot)
{
    if (a.narrow) {
        const uint32_t group = id / (8 * a.Hkv), r = id % (8 * a.Hkv);
        kvh = r >> 3;
        slot = a.slots - 1 - static_cast<int>(group * 8 + (r & 7));
    } else {
        kvh = id % a.Hkv;
        slot = a.slots - 1 - static_cast<int>(id / a.Hkv);
    }
}

// the lanes of a wave, for the search of a block's sequence
struct WaveLanes {
    int v;
    template <typename F> __device__ __forceinline__ uint64_t probe(F f)
    {
        const Probe p = f(static_cast<int>(threadIdx.x & 63));
        v = p.value;
        return __ballot(p.ok);
    }
    __device__ __forceinline__ int value(int c) const { return __builtin_amdgcn_readlane(v, c); }
    __device__ __forceinline__ static int uniform(int x)
    {
        return __builtin_amdgcn_readfirstlane(x);
    }
};
template <int TR>
__device__ __forceinline__ Span find_span(const int *start, int S, int T, int G, int w)
{
    WaveLanes lanes;
    return find_span<TR>(lanes, start, S, T, G, w);
}

} // namespace attn
} // namespace hexk
