// Which kernel takes a product in 8 bits: rules on its sizes alone.  Plain C++ without device code, so that a host program can ask too.
#pragma once
#include "gemm_plan.h"

namespace tfla {

// Whether a pair's kernel forms h and its codes: a tile of 256 x 256 holds the 128 columns of a scale, all of their contraction.
inline bool q8_gate_inside(int bn, int split) { return bn == 256 && split == 1; }

// ---- the quantiser's tiles ------------------------------------------------------------------------
// A workgroup of 1024 threads per tile of 128 x 128.  The runtime starts fewer than 2^32 threads along an axis, and matrices of 2^36 values have
// 2^22 tiles: what is more than Q8_LAUNCH workgroups follows in further launches (a multiple of eight, so that workgroup i of all of them goes on
// running on XCD i % 8).
constexpr int Q8_TILE = 128, Q8_TILE_THREADS = 1024;
constexpr unsigned Q8_LAUNCH = 1u << 21;
inline unsigned q8_tiles(long M, long N) { return (unsigned)((M + Q8_TILE - 1) / Q8_TILE * ((N + Q8_TILE - 1) / Q8_TILE)); }
// workgroups of the launch that begins with workgroup `first` of `all`
inline unsigned q8_launch(unsigned first, unsigned all) { return all - first < Q8_LAUNCH ? all - first : Q8_LAUNCH; }

// ---- tiles of products ------------------------------------------------------------------------------
// How a product is cut: the tile and the number of parts with the shortest time by a model as gemm_plan's, with steps of 128 codes.  Fitted to
// 2500 times of 260 random products (33 to 8192 rows, 64 to 8192 columns, contractions of 128 to 8192; pairs, two segments, two at a
// time): 8 % off in the mean, and what it picks is 1.3 % above the best of all choices on average, 23 % at most.  In us:
//   256 x 256   8.7 + n (t (0.97 + 0.43 min(1, w / 256)) + 4.6)      (a pair with its gate inside: 11.2 in place of 4.6)
//   256 x 128   6.6 + n (t (0.66 + 0.16 min(1, w / 256)) + 4.5)
//   128 x 128   6.1 + t (0.43 + 0.28 w / 256) up to 256 workgroups, 7 + n (0.45 t + 0.5) + 1.5 max(0, n - 2) above
//   64 x 64     5.6 + 0.193 t n + 1.2 max(0, n - 2)                  (pairs: 64 x 128, 0.396 t n)
//   joining the parts, or a pair's gate outside   3.1 + (bytes written and read again) / 7 MB per us
inline GemmPlan q8_plan(long M, int N, int K, int segs, int batch, int pair) {
    struct Tile { int bm, bn; };
    static constexpr Tile tiles[] = {{256, 256}, {256, 128}, {128, 128}, {64, 64}};
    const int step = 128, all = (K + step - 1) / step * segs;
    GemmPlan best{};
    for (const Tile& tile : tiles) {
        const int bm = tile.bm, bn = pair && bm == 64 ? 128 : tile.bn, bno = pair ? bn / 2 : bn;
        const double cells = (double)((M + bm - 1) / bm) * ((N + bno - 1) / bno) * batch;
        for (int split = 1; split <= 32 && (split == 1 || (all >= 4 * split && cells * split <= 1024)); split += split < 4 ? 1 : split / 2) {
            const double w = cells * split, t = (all + split - 1) / split, part = w < 256 ? w / 256 : 1, n = (double)(long)((w + 255) / 256);
            const double more = n > 2 ? n - 2 : 0;
            const bool inside = pair && q8_gate_inside(bn, split);
            double us;
            if (bn == 256) us = 8.7 + n * (t * (0.97 + 0.43 * part) + (inside ? 11.2 : 4.6));
            else if (bm == 256) us = 6.6 + n * (t * (0.66 + 0.16 * part) + 4.5);
            else if (bm == 128) us = n < 2 ? 6.1 + t * (0.43 + 0.28 * part) : 7 + n * (0.45 * t + 0.5) + 1.5 * more;
            else us = 5.6 + (pair ? 0.396 : 0.193) * t * n + 1.2 * more;
            if (split > 1 || (pair && !inside)) us += 3.1 + 8.0 * split * (pair ? 2 : batch) * (double)M * N / 7e6;
            if (best.bm == 0 || us < best.us) best = {bm, bn, split, us};
        }
    }
    return best;
}

// ---- both products of a small backward pass in one launch ------------------------------------------
// dx and dw in tiles of 64 x 64, undivided, and the bias gradients' sums with them: a launch saved (3.4 us of the host's time, 2 of the GPU's; two
// with sums), and the items of one product fill what the other leaves of the CUs' time, where by an estimate that is no slower.  (Weights of close to
// 2^36 elements with a few tokens are 2^24 tiles of 256 threads, 2^32: the runtime does not start that many, two products of larger tiles do.)
inline bool q8_both_applies(const GemmPlan& x, const GemmPlan& w, long M, int K, int N, int pair) {
    auto up = [](long v, int by) { return (v + by - 1) / by; };
    const long segs = pair ? 2 : 1, nx = up(M, 64) * up(K, 64), nw = up(N, 64) * up(K, 64) * segs, tx = up(N, 128) * segs, tw = up(M, 128);
    if ((nx + nw + up(N * segs, 256)) * 256 >> 32) return false;
    const double share = (nx * tx + nw * tw) / 256.0, longest = tx > tw ? tx : tw, chain = (nx + nw > 256 ? 0.4 : 0.2) * longest;
    const double us = 7.5 + (0.31 * share > chain ? 0.31 * share : chain);
    return us <= x.us + w.us + 2;
}

// ---- few rows -----------------------------------------------------------------------------------
constexpr int Q8_ROWS_MAX = 32;
// Slices as in gemm_plan.h, wherever the rows of x leave room for them: a block of work is 16 / slices rows of weights (one token through
// 10944 x 4096 11.3 us, in one slice 14.3, 8 tokens 13.3 and 15.2; through 4096 x 4096, where the host's time is most of it, 7.2 and 7.3,
// 7.9 and 7.9; 4 tokens there 7.8 and 7.6).  A slice's pieces of
// 128 codes go round the wavefronts, `ahead` of them per wavefront in flight, so that few places stay empty: a place without a piece costs
// what one with a piece does (4 tokens through a pair of 10944 x 4096, 8 pieces a slice: four wavefronts with two pieces 18.4 us, with four
// 37.2; through 4096 x 10944, 22 pieces: eight wavefronts with one 11.0, with two 13.3).  hold: a wavefront's share of x is one turn, and
// there are more blocks than the chip runs at a time.
struct Q8RowsPlan { int row_blocks, slices, waves, ahead, blocks, grid; bool hold; };
inline Q8RowsPlan q8_rows_plan(long M, int N, int K, int pair) {
    Q8RowsPlan p{};
    p.row_blocks = M <= 16 ? 1 : 2;
    p.slices = M <= 4 ? 4 : (M <= 8 ? 2 : 1);
    p.blocks = (N + 16 / p.slices - 1) / (16 / p.slices);
    const int pieces = ((K + 127) / 128 + p.slices - 1) / p.slices;
    p.waves = pieces < 16 ? 4 : (pieces >= 32 && p.blocks <= 256 ? 16 : 8);
    const int one = (pieces + p.waves - 1) / p.waves, two = (pieces + 2 * p.waves - 1) / (2 * p.waves);
    p.ahead = 2 * two <= one ? 2 : 1;
    const int most = 256 * (p.waves == 4 ? 4 : 2);
    p.hold = p.waves <= 8 && p.ahead == 2 && two == 1 && p.blocks > most;
    // three turns as one, x held: 4 tokens through 10944 x 5504 17.9 us, so 14.4; not where x is a row or two (13.3, 14.7), for pairs (28.3, 30.8), where
    // the slices lack more than two pieces (10944 x 4104: 15.3, 18.4) or blocks are few (4096 x 10944: 10.9, 12.0)
    const int all = (K + 127) / 128;
    if (p.slices == 4 && M > 2 && !pair && p.waves <= 8 && one == 3 && p.blocks > 2 * most && 4 * pieces - all <= 2) { p.ahead = 3; p.hold = true; }
    p.grid = p.hold ? most : p.blocks;
    return p;
}
// Whether this kernel takes a product or the tiles do: by estimates of both, here rounds of blocks at 30 GB/s per CU (one round: 39).  Calls,
// here and there: 4096 x 4096, 8 rows 8.2 and 10.7 us, 32 rows 9.5 and 10.8; 4096 x 10944, 32 rows 15.5 and 14.4; pair of 10944 x 4096, 8
// rows 22.5 and 22.2, 16 rows 28.7 and 22.5.  copies: operands that the tiles cannot read in place.
inline bool q8_rows_applies(long M, int N, int K, int pair, bool copies) {
    if (M <= 4 || M > Q8_ROWS_MAX) return M <= 4;
    if (copies) return true;
    const Q8RowsPlan p = q8_rows_plan(M, N, K, pair);
    const double bytes = (double)(16 / p.slices * (pair ? 2 : 1) + M) * K;
    const double here = 1.8 + (p.blocks + 255) / 256 * bytes / (p.blocks <= 256 ? 39e3 : 30e3) + (pair ? 3.1 : 0);
    return here <= q8_plan(M, N, K, 1, 1, pair).us;
}

}  // namespace tfla
