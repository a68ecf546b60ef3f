// gemm_plan_query.cpp -- exposes the matrix products' division among blocks
// (paper_1903_01814_amd/csrc/gemm_plan.h, host arithmetic only) to the CPU tests
// through a C interface.  Built with g++ by the tests.
#include "gemm_plan.h"

#include <initializer_list>

namespace hexk {
static int g_cus = 256;
int device_cus() { return g_cus; }
} // namespace hexk

extern "C" {

void set_cus(int n) { hexk::g_cus = n; }

// out: parts, bytes of split sums, then per part: tile, first, rows, mt, nt, steps,
// splits, per
void gemm_plan_query(int M, int N, int K, int gated, int planes, long *out)
{
    const hexk::gemm::Plan p = hexk::gemm::make_plan(M, N, K, gated != 0, planes);
    *out++ = p.parts;
    *out++ = static_cast<long>(hexk::gemm::part_bytes(p, gated != 0));
    for (int i = 0; i < p.parts; ++i) {
        const hexk::gemm::Part &q = p.part[i];
        for (long v : {(long)q.tile, (long)q.first, (long)q.rows, (long)q.mt, (long)q.nt,
                       (long)q.steps, (long)q.splits, (long)q.per})
            *out++ = v;
    }
}
}
