// Which kernel takes a product in 8 bits: rules on its sizes alone.  Plain C++ without device code, so that a host program can ask too.
#pragma once
#include "gemm_plan.h"

namespace tfla {

// Tiles of 256 x 256 to 64 x 64 (pairs: 64 x 128); a step of the contraction is 128 codes.
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
            double us;
            if (bn == 256) us = 8 + n * (t * (1.0 + 0.45 * part) + 4);
            else if (bm == 256) us = 7 + n * (t * (0.63 + 0.31 * part) + 2);
            else if (bm == 128) us = n < 2 ? 5 + t * (0.42 + 0.15 * part) : 6 + 0.49 * t * n + 1.5 * more;
            else us = 4.8 + (pair ? 0.34 : 0.177) * t * n + 0.9 * more;
            if (split > 1) us += 4.2 + 8.0 * split * (pair ? 2 : batch) * (double)M * N / 7e6;
            if (best.bm == 0 || us < best.us) best = {bm, bn, split, us};
        }
    }
    return best;
}
// Whether a pair's kernel forms h and its codes: a tile of 256 x 256 holds the 128 columns of a scale, all of their contraction.
inline bool q8_gate_inside(const GemmPlan& p) { return p.bn == 256 && p.split == 1; }

// ---- few rows -----------------------------------------------------------------------------------
constexpr int Q8_ROWS_MAX = 32;
inline bool q8_rows_applies(long M) { return M <= Q8_ROWS_MAX; }
// Slices as in gemm_plan.h, wherever the rows of x leave room for them: a block of work is 16 / slices rows of weights.  A slice's pieces of
// 128 codes go round the wavefronts, `ahead` of them per wavefront in flight, so that few places stay empty: a place without a piece costs
// what one with a piece does (4 tokens through a pair of 10944 x 4096, 8 pieces a slice: four wavefronts with two pieces 18.4 us, with four
// 37.2; through 4096 x 10944, 22 pieces: eight wavefronts with one 11.0, with two 13.3).  hold: a wavefront's share of x is one turn, and
// there are more blocks than the chip runs at a time.
struct Q8RowsPlan { int row_blocks, slices, waves, ahead, blocks, grid; bool hold; };
inline Q8RowsPlan q8_rows_plan(long M, int N, int K) {
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
    p.grid = p.hold ? most : p.blocks;
    return p;
}

}  // namespace tfla
