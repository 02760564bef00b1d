// How many threads the residual block's calls start at once, by the rules that the library itself is built with.  Compiled by the tests with the host
// compiler.
#include "q8_plan.h"

using namespace tfla;

static long largest(long a, long b) { return a > b ? a : b; }
static long threads_of(const GemmPlan& p, long M, int N, int batch, int pair) {
    const long n = gemm_workgroups(p, M, N, batch, pair);
    return p.bm == 256 ? 256 * 256 : n * (gemm_many(n) ? 256 : 512);
}

// threads of the largest launch of a call's products (the wide kernels start 256 workgroups at most)
extern "C" long product_threads(int backward, int pair, long M, int K, int N) {
    if (!backward) {
        if (q8_rows_applies(M, N, K, pair, true)) {
            const Q8RowsPlan p = q8_rows_plan(M, N, K, pair);
            return (long)p.blocks * p.waves * 64;
        }
        const GemmPlan p = q8_plan(M, N, K, 1, 1, pair);
        return largest(threads_of(p, M, N, 1, pair), pair ? (M + 3) / 4 * 256 : 0);        // (a pair's gate: four rows a workgroup)
    }
    const int P = pair ? 2 : 1;
    const GemmPlan x = q8_plan(M, K, N, P, 1, 0), w = q8_plan(N, K, M, 1, P, 0);
    if (q8_both_applies(x, w, M, K, N, pair)) {
        const long up_m = (M + 63) / 64, up_k = (K + 63) / 64, up_n = (N + 63) / 64, n = up_m * up_k + up_n * up_k * P;
        const long threads = gemm_many(n) ? 256 : 512;
        return (n + ((long)P * N + threads - 1) / threads) * threads;
    }
    return largest(threads_of(x, M, K, 1, 0), threads_of(w, N, K, P, 0));
}

// launches of the quantiser's tiles with `more` workgroups behind them: first workgroup and threads of each; their number
extern "C" int tile_launches(long M, long N, unsigned more, long* first, long* threads) {
    const unsigned all = q8_tiles(M, N) + more;
    int n = 0;
    for (unsigned at = 0; at < all; at += q8_launch(at, all)) {
        first[n] = at;
        threads[n++] = (long)q8_launch(at, all) * Q8_TILE_THREADS;
    }
    return n;
}

// work items of 256 threads of a backward call's products in one launch, those of bf16; 0: two launches
extern "C" long both_items(int pair, long M, int K, int N) {
    const GemmPlan x = gemm_plan(M, K, N, pair ? 2 : 1, 1, 0, 1), w = gemm_plan(N, K, M, 1, pair ? 2 : 1, 0, 1);
    return gemm_both_applies(x, w, M, K, N, pair, 1) ? both_steps(M, K, N, pair).items : 0;
}
