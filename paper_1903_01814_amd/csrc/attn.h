// attn.h -- what the attention kernels share: matrix-core operands of either
// type, the LDS layout of a staged tile, the walk over packed sequences.
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

#include "hexdev.h"
#include "kernels.h"

namespace hexk {
namespace attn {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));

// log2(e) and ln(2) as a float and what it leaves
constexpr float kLog2e = 1.4426950408889634f, kLog2eLo = 1.4426950408889634 - kLog2e;
constexpr float kLn2 = 0.6931471805599453f, kLn2Lo = 0.6931471805599453 - kLn2;

constexpr int kShortRows = 256;

struct FragF32 {
    float v[8];
};

template <typename E> struct Elem;
template <> struct Elem<bf16raw> {
    using Frag = bf16x8;
    static constexpr int VEC = 8; // elements of a 16-byte vector
};
template <> struct Elem<float> {
    using Frag = FragF32;
    static constexpr int VEC = 4;
};

__device__ __forceinline__ floatx16 mma(bf16x8 a, bf16x8 b, floatx16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ floatx16 mma(const FragF32 &a, const FragF32 &b, floatx16 c)
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[i], b.v[i], c, 0, 0, 0);
    return c;
}

// The next 16 elements of a sum over the head dimension.  float32: the
// matrix core adds them from zero and the vector unit adds that to the sum, so
// that a score of D = 128 is 8 roundings of its own size and not 64 (scores of
// 100, whose exponentials carry 100 times a score's relative error: a third
// of it; the additions run beside the next products).
__device__ __forceinline__ floatx16 add_product(bf16x8 a, bf16x8 b, floatx16 c)
{
    return mma(a, b, c);
}
__device__ __forceinline__ floatx16 add_product(const FragF32 &a, const FragF32 &b, floatx16 c)
{
    return c + mma(a, b, floatx16{});
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
template <typename E>
__device__ __forceinline__ float prob(float x, const AttnArgs &a, float hi, float lo)
{
    float e = fmaf(x, a.c, -hi);
    if constexpr (sizeof(E) == 4)
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
template <typename E> __device__ __forceinline__ typename Elem<E>::Frag to_frag(const floatx16 &x, int s)
{
    if constexpr (sizeof(E) == 2) {
        bf16x8 f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = static_cast<__bf16>(x[8 * s + i]);
        return f;
    } else {
        FragF32 f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f.v[i] = x[8 * s + i];
        return f;
    }
}

// ---- tiles in LDS: rows of DC head elements (a multiple of 32, padded with
// zeros), 16-byte chunks permuted within the row by its number, so that both
// reads below spread over all 64 banks: sixteen rows of one chunk
// (read_cols), and runs of 64 or 128 bytes of four to eight rows (read_rows).
template <typename E, int DC> struct Tile {
    static constexpr int PITCH = (DC == 96 ? 128 : DC) * static_cast<int>(sizeof(E)); // bytes a row
    static constexpr int CPR = DC * static_cast<int>(sizeof(E)) / 16; // chunks in use
    static constexpr int bytes(int rows) { return rows * PITCH; }

    __device__ __forceinline__ static int swz(int row)
    {
        if constexpr (sizeof(E) == 2) {
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
        return row * PITCH + (((sizeof(E) == 2 ? h : 2 * h) ^ swz(row)) << 4);
    }
    __device__ __forceinline__ static typename Elem<E>::Frag read_cols(const unsigned char *t,
                                                                       int at, int s)
    {
        if constexpr (sizeof(E) == 2) {
            return *reinterpret_cast<const bf16x8 *>(t + (at ^ (s << 5)));
        } else {
            FragF32 f;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 u = *reinterpret_cast<const float4 *>(t + (at ^ (s << 6 | j << 4)));
                f.v[4 * j] = u.x, f.v[4 * j + 1] = u.y, f.v[4 * j + 2] = u.z, f.v[4 * j + 3] = u.w;
            }
            return f;
        }
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
        if constexpr (sizeof(E) == 2) {
            const int r = 4 * h + ((lane & 15) >> 2);
            const int c = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), o = 8 * (lane & 1);
            return RowsAt{chunk_at(r, c) + o, chunk_at(r + 8, c) + o};
        } else {
            return RowsAt{chunk_at(4 * h, (lane & 31) >> 2) + 4 * (lane & 3), 0};
        }
    }
    __device__ __forceinline__ static typename Elem<E>::Frag read_rows(unsigned char *t, RowsAt at,
                                                                       int row0, int d)
    {
        if constexpr (sizeof(E) == 2) {
            using lp = __attribute__((address_space(3))) shortx4 *;
            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lp)(t + row0 * PITCH + (at.a ^ (d << 6))));
            const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lp)(t + row0 * PITCH + (at.b ^ (d << 6))));
            return __builtin_bit_cast(bf16x8,
                                      __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            // the permutation of row 8 (i / 4) + 4 h + i % 4 is that of row 4 h
            // and that of the rest, by exclusive or
            FragF32 f;
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

// One operand of 8 head elements from global memory, zeros past D; `p` is the
// row's start (16-byte aligned), c the first element (a multiple of 8, as D).
template <typename E>
__device__ __forceinline__ typename Elem<E>::Frag load_frag(const E *p, int c, int D)
{
    if constexpr (sizeof(E) == 2) {
        uint4 u{0, 0, 0, 0};
        if (c < D)
            u = *reinterpret_cast<const uint4 *>(p + c);
        return __builtin_bit_cast(bf16x8, u);
    } else {
        FragF32 f;
        float4 u{0, 0, 0, 0}, w{0, 0, 0, 0};
        if (c < D) {
            u = *reinterpret_cast<const float4 *>(p + c);
            w = *reinterpret_cast<const float4 *>(p + c + 4);
        }
        f.v[0] = u.x, f.v[1] = u.y, f.v[2] = u.z, f.v[3] = u.w;
        f.v[4] = w.x, f.v[5] = w.y, f.v[6] = w.z, f.v[7] = w.w;
        return f;
    }
}

__device__ __forceinline__ float dot8(const FragF32 &a, const FragF32 &b)
{
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        s = fmaf(a.v[i], b.v[i], s);
    return s;
}
__device__ __forceinline__ float dot8(bf16x8 a, bf16x8 b)
{
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        s = fmaf(static_cast<float>(a[i]), static_cast<float>(b[i]), s);
    return s;
}

// ---- packed sequences ----------------------------------------------------
// The rows of one (sequence, key head) are its query tokens times the G query
// heads that share the key head, heads fastest.  Work is handed out in tiles
// of TR rows.  Sequence s owns tile slots start[s] G / TR + s up to the next
// sequence's first, which is as many as it needs or one more; so the slots
// are known without the lengths on the host, rows G / TR + S in all.

// token of row r: r / G by the reciprocal, which gives it or one less
__device__ __forceinline__ int row_token(Group g, int r)
{
    const uint32_t t = __umulhi(static_cast<uint32_t>(r), g.inv);
    return static_cast<int>(t + (static_cast<uint32_t>(r) - t * g.G >= static_cast<uint32_t>(g.G)));
}

inline int attn_slots(int T, int G, int TR, int S)
{
    return static_cast<int>(static_cast<int64_t>(T) * G / TR) + S;
}
// Sequences too short to fill tiles of 128 rows: tiles of 64
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

__device__ __forceinline__ int clamp_start(const int *start, int i, int T)
{
    return min(max(start[i], 0), T);
}

// One tile on its way from memory to LDS: ROWS rows, a 16-byte chunk a thread
// at a time, NT threads.  Addresses are a uniform base and a 32-bit offset
// (token strides are below 2^24 bytes), so that a load costs two or three
// vector instructions beside itself.  Chunks past D stay zero.
template <typename E, int DC, int ROWS, int NT> struct Stage {
    using TL = Tile<E, DC>;
    static constexpr int N = ROWS * TL::CPR / NT;
    static_assert(ROWS * TL::CPR % NT == 0, "");
    uint4 r[N];

    __device__ __forceinline__ Stage()
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
            r[i] = uint4{0, 0, 0, 0};
    }
    __device__ __forceinline__ static int row(int i) { return (threadIdx.x % NT + NT * i) / TL::CPR; }
    __device__ __forceinline__ static int chunk(int i) { return (threadIdx.x % NT + NT * i) % TL::CPR; }
    __device__ __forceinline__ void get(int i, const E *base, uint32_t bytes, int D)
    {
        if (chunk(i) * Elem<E>::VEC < D)
            r[i] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(base) + bytes);
    }
    // rows from `base` on, ld bytes apart; those past the last of `left`
    // repeat it
    __device__ __forceinline__ void rows(const E *base, uint32_t ld, int left, int D)
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
            get(i, base, __umul24(min(row(i), left - 1), ld) + 16 * chunk(i), D);
    }
    __device__ __forceinline__ void put(unsigned char *t) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
            *reinterpret_cast<uint4 *>(t + TL::chunk_at(row(i), chunk(i))) = r[i];
    }
};

// Which (key head, tile slot) block `id` takes.  Dies take blocks in turn, 8 of
// them.  Usually key heads are innermost, so that a head's keys stay on few
// dies.  Heads of less than a 128-byte cache line share lines with their
// neighbours: there all heads of a slot go to one die (512 sequences of 20 to
// 400 tokens, 8 heads of 32 bf16 elements: see attn_fwd_k).  Slots from the
// last on: under the causal mask a sequence's last tiles are the longest.
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

struct Span {
    int seq;      // sequence
    int begin, n; // its tokens
    int tile;     // which of its tiles
};

// Sequence that owns tile slot w: 64 probes at once, log_64(S) rounds, the
// last of which leaves the neighbouring offsets in the lanes.
template <int TR>
__device__ __forceinline__ Span find_span(const int *start, int S, int T, int G, int w)
{
    const int lane = threadIdx.x & 63;
    auto slot = [&](int v, int i) {
        return static_cast<int>(static_cast<int64_t>(v) * G / TR) + i;
    };
    int lo = 0, n = S, v, c;
    for (;;) {
        const int step = (n + 63) >> 6, at = lo + lane * step;
        // one probe past the last, for the sequence's end
        v = clamp_start(start, min(at, S), T);
        const bool ok = lane * step < n && slot(v, at) <= w;
        c = max(1, __popcll(__ballot(ok))) - 1;
        lo += c * step;
        if (step == 1)
            break;
        n = min(step, n - c * step);
    }
    Span s;
    s.seq = __builtin_amdgcn_readfirstlane(lo);
    c = __builtin_amdgcn_readfirstlane(c);
    s.begin = __builtin_amdgcn_readlane(v, c);
    const int end = c < 63 ? __builtin_amdgcn_readlane(v, c + 1) : clamp_start(start, s.seq + 1, T);
    s.n = max(0, end - s.begin);
    s.tile = w - slot(s.begin, s.seq);
    return s;
}

} // namespace attn
} // namespace hexk
