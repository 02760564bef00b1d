// The kernels that a call of the residual block's products launches, by the rules that the library itself is built with: a line per
// launch.  Compiled by the tests with the host compiler.
#include "gemm_plan.h"

#include <cstdio>
#include <cstring>

using namespace tfla;

static int tile(char* to, const char* what, int dtype, int pair, const GemmPlan& p, long workgroups) {
    return sprintf(to, "%s %s%s %dx%d%s%s\n", what, dtype ? "bf16" : "fp32", pair ? " pair" : "", p.bm, p.bn, p.split > 1 ? " divided" : "",
                   gemm_many(workgroups) ? " many" : "");
}

// backward: 0 or 1; dtype: 0 fp32, 1 bf16; tensors at multiples of 16 bytes.  Returns the launches' names in `to`.
extern "C" void product_kernels(int backward, int dtype, int pair, long M, int K, int N, char* to) {
    *to = 0;
    if (!backward) {
        const bool copies = dtype == 1 && K % 8 != 0;
        if (gemm_rows_applies(M, N, K, pair, dtype, copies)) {
            const RowsPlan p = rows_plan(M, N, K, pair, dtype ? 2 : 4);
            sprintf(to, "rows %s%s blocks %d slices %d waves %d%s\n", dtype ? "bf16" : "fp32", pair ? " pair" : "", p.row_blocks, p.slices, p.waves,
                    p.hold ? " hold" : "");
            return;
        }
        const GemmPlan p = gemm_plan(M, N, K, 1, 1, pair, dtype);
        tile(to, "fwd", dtype, pair, p, gemm_workgroups(p, M, N, 1, pair));
        return;
    }
    const GemmPlan x = gemm_plan(M, K, N, pair ? 2 : 1, 1, 0, dtype), w = gemm_plan(N, K, M, 1, pair ? 2 : 1, 0, dtype);
    if (gemm_both_applies(x, w, M, K, N, pair, dtype)) {
        const BothSteps b = both_steps(M, K, N, pair);
        if (dtype == 1) sprintf(to, "both bf16%s %s\n", pair ? " pair" : "", b.wide() ? "64x128" : (gemm_many(b.items) ? "64x64 many" : "64x64"));
        else sprintf(to, "both fp32%s %dx%d\n", pair ? " pair" : "", x.bm, x.bn);
        return;
    }
    to += tile(to, "dx", dtype, pair, x, gemm_workgroups(x, M, K, 1, 0));
    tile(to, "dw", dtype, pair, w, gemm_workgroups(w, N, K, pair ? 2 : 1, 0));
}
