// attn_span.h -- which rows of which sequence a block of the attention kernels
// takes: integer arithmetic only, with the lanes of a wave as a parameter, so
// that it also compiles with a plain C++ compiler and can be checked without a
// GPU.
//
// The rows of one (sequence, key head) are its query tokens times the G query
// heads that share the key head, heads fastest.  Work is handed out in tiles
// of TR rows.  Sequence s owns tile slots start[s] G / TR + s up to the next
// sequence's first, which is as many as it needs or one more; so the slots
// are known without the lengths on the host, rows G / TR + S in all.
#pragma once

#include <stdint.h>

#include "hexgeom.h"

namespace hexk {

// Query heads that share a key head, and the reciprocal that divides by their
// number: floor(2^32 / G) (2^32 - 1 for G = 1) times r, shifted down, is r / G
// or one less for every r < 2^31.
struct Group {
    int G;
    uint32_t inv;
};
inline Group make_group(int G)
{
    return {G, G == 1 ? 0xffffffffu : static_cast<uint32_t>((1ull << 32) / G)};
}

namespace attn {

// token of row r >= 0: r / G by the reciprocal, which gives it or one less
HEX_HD int row_token(Group g, int r)
{
    const uint32_t u = static_cast<uint32_t>(r);
    const uint32_t t = static_cast<uint32_t>(static_cast<uint64_t>(u) * g.inv >> 32);
    return static_cast<int>(t + (u - t * g.G >= static_cast<uint32_t>(g.G)));
}

inline int attn_slots(int T, int G, int TR, int S)
{
    return static_cast<int>(static_cast<int64_t>(T) * G / TR) + S;
}

// offset i, brought into the tensor
HEX_HD int clamp_start(const int *start, int i, int T)
{
    const int v = start[i];
    return v < 0 ? 0 : v < T ? v : T;
}

struct Span {
    int seq;      // sequence
    int begin, n; // its tokens
    int tile;     // which of its tiles
};

// What a lane found at its probe.
struct Probe {
    int value; // an offset
    bool ok;
};

// Sequence that owns tile slot w: 64 probes at once, log_64(S) rounds, the
// last of which leaves the neighbouring offsets in the lanes.  Whatever the
// offsets are, rows tile TR .. of the n G lie inside the tensor.
//
// Lanes: `probe(f)` runs f(lane) -> Probe in 64 lanes, keeps the values and
// returns the lanes that were ok as bits; `value(c)` is lane c's value;
// `uniform(v)` says that v is the same in all lanes.
template <int TR, typename Lanes>
HEX_HD Span find_span(Lanes &lanes, const int *start, int S, int T, int G, int w)
{
    auto slot = [&](int v, int i) {
        return static_cast<int>(static_cast<int64_t>(v) * G / TR) + i;
    };
    int lo = 0, n = S, c;
    for (;;) {
        const int step = (n + 63) >> 6;
        const uint64_t ok = lanes.probe([&](int lane) {
            // one probe past the last, for the sequence's end
            const int at = lo + lane * step, v = clamp_start(start, at < S ? at : S, T);
            return Probe{v, lane * step < n && slot(v, at) <= w};
        });
        const int found = __builtin_popcountll(ok);
        c = found > 1 ? found - 1 : 0;
        lo += c * step;
        if (step == 1)
            break;
        n = step < n - c * step ? step : n - c * step;
    }
    Span s;
    s.seq = lanes.uniform(lo);
    c = lanes.uniform(c);
    s.begin = lanes.value(c);
    const int end = c < 63 ? lanes.value(c + 1) : clamp_start(start, s.seq + 1, T);
    s.n = end > s.begin ? end - s.begin : 0;
    s.tile = w - slot(s.begin, s.seq);
    // Slots before the first sequence's own, and some of offsets that do not
    // ascend, belong to no sequence: no rows.
    if (s.tile < 0)
        s.n = s.tile = 0;
    return s;
}

} // namespace attn
} // namespace hexk
