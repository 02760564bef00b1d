// How many threads the calls in 8 bits start at once, by the rules that the library itself is built with.  Compiled by the tests with the host
// compiler.
#include "q8_plan.h"

using namespace tfla;

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
