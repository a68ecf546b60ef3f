// attn_rows.cpp -- replays on the CPU which rows the attention kernels' blocks
// take (paper_1903_01814_amd/csrc/attn_span.h): every tile slot of a call, with
// an array in place of a wave's lanes.  Built with g++ by the tests.
#include "attn_span.h"

namespace {

struct ArrayLanes {
    int v[64];
    template <typename F> uint64_t probe(F f)
    {
        uint64_t ok = 0;
        for (int i = 0; i < 64; ++i) {
            const hexk::attn::Probe p = f(i);
            v[i] = p.value;
            ok |= static_cast<uint64_t>(p.ok) << i;
        }
        return ok;
    }
    int value(int c) const { return v[c]; }
    static int uniform(int x) { return x; }
};

int clamp(int v, int T) { return v < 0 ? 0 : v < T ? v : T; }

template <int TR> long replay(const int *start, int S, int T, int G, int *taken)
{
    long outside = 0;
    const hexk::Group g = hexk::make_group(G);
    const int slots = hexk::attn::attn_slots(T, G, TR, S);
    for (int w = 0; w < slots; ++w) {
        ArrayLanes lanes;
        const hexk::attn::Span sp = hexk::attn::find_span<TR>(lanes, start, S, T, G, w);
        if (sp.seq < 0 || sp.seq >= S) {
            ++outside;
            continue;
        }
        const int rows = sp.n * G;
        // the kernels leave here
        if (static_cast<int64_t>(sp.tile) * TR >= rows)
            continue;
        const int row0 = sp.tile * TR;
        const int begin = clamp(start[sp.seq], T), end = clamp(start[sp.seq + 1], T);
        for (int i = 0; i < TR; ++i) {
            const int row = row0 + i, rc = row < rows ? row : rows - 1;
            const int64_t tq = hexk::attn::row_token(g, rc), head = rc - tq * G;
            const int64_t token = sp.begin + tq;
            if (token < begin || token >= end || head < 0 || head >= G)
                ++outside;
            else if (row < rows)
                ++taken[token * G + head];
        }
    }
    return outside;
}

} // namespace

extern "C" {

// Adds one to taken[token G + head] for every row that a block takes; returns
// how many rows lie outside their sequence.
long attn_rows(const int *start, int S, int T, int G, int TR, int *taken)
{
    return TR == 64 ? replay<64>(start, S, T, G, taken) : replay<128>(start, S, T, G, taken);
}
}
