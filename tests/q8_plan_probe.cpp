// The kernels that a call of the products in 8 bits launches, by the rules that the library itself is built with: a line per launch of a
// product.  Compiled by the tests with the host compiler.
#include "q8_plan.h"

#include <cstdio>

using namespace tfla;

static int tile(char* to, const char* what, int pair, const GemmPlan& p, long workgroups) {
    return sprintf(to, "%s%s %dx%d%s%s\n", what, pair ? " pair" : "", p.bm, p.bn, p.split > 1 ? " divided" : "", gemm_many(workgroups) ? " many" : "");
}

// operands at multiples of 16 bytes
extern "C" void product_kernels(int backward, int pair, long M, int K, int N, char* to) {
    *to = 0;
    if (!backward) {
        if (q8_rows_applies(M, N, K, pair, K % 16 != 0)) {
            const Q8RowsPlan p = q8_rows_plan(M, N, K, pair);
            const bool odd = K % 4 != 0;
            sprintf(to, "rows%s blocks %d slices %d waves %d ahead %d%s\n", pair ? " pair" : "", p.row_blocks, p.slices, p.waves,
                    odd && p.ahead == 3 ? 1 : p.ahead, odd ? " odd" : (p.hold ? " hold" : ""));
            return;
        }
        const GemmPlan p = q8_plan(M, N, K, 1, 1, pair);
        tile(to, "fwd", pair, p, gemm_workgroups(p, M, N, 1, pair));
        return;
    }
    const GemmPlan x = q8_plan(M, K, N, pair ? 2 : 1, 1, 0), w = q8_plan(N, K, M, 1, pair ? 2 : 1, 0);
    if (q8_both_applies(x, w, M, K, N, pair)) {
        const long up_m = (M + 63) / 64, up_k = (K + 63) / 64, up_n = (N + 63) / 64;
        sprintf(to, "both%s%s\n", pair ? " pair" : "", gemm_many(up_m * up_k + up_n * up_k * (pair ? 2 : 1)) ? " many" : "");
        return;
    }
    to += tile(to, "dx", pair, x, gemm_workgroups(x, M, K, 1, 0));
    tile(to, "dw", pair, w, gemm_workgroups(w, N, K, pair ? 2 : 1, 0));
}
