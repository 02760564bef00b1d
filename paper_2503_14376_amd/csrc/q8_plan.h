// Which kernel takes a product in 8 bits: rules on its sizes alone.  Plain C++ without device code, so that a host program can ask too.
#pragma once
#include "gemm_plan.h"

namespace tfla {

// Tiles of 128 x 128 or 64 x 64 (pairs: 64 x 128); a step of the contraction is 128 codes.
inline GemmPlan q8_plan(long M, int N, int K, int segs, int batch, int pair) {
    const int step = 128, all = (K + step - 1) / step * segs;
    GemmPlan best{};
    for (int bm : {128, 64}) {
        const int bn = pair && bm == 64 ? 128 : bm, bno = pair ? bn / 2 : bn;
        const double cells = (double)((M + bm - 1) / bm) * ((N + bno - 1) / bno) * batch;
        for (int split = 1; split <= 32 && (split == 1 || (all >= 4 * split && cells * split <= 1024)); split += split < 4 ? 1 : split / 2) {
            const double w = cells * split, t = (all + split - 1) / split, part = w < 256 ? w / 256 : 1, n = (double)(long)((w + 255) / 256);
            const double more = n > 2 ? n - 2 : 0;
            double us = bm == 128 ? (n < 2 ? 5 + t * (0.42 + 0.15 * part) : 6 + 0.49 * t * n + 1.5 * more) : 4.8 + (pair ? 0.34 : 0.177) * t * n + 0.9 * more;
            if (split > 1) us += 4.2 + 8.0 * split * (pair ? 2 : batch) * (double)M * N / 7e6;
            if (best.bm == 0 || us < best.us) best = {bm, bn, split, us};
        }
    }
    return best;
}

// ---- few rows -----------------------------------------------------------------------------------
constexpr int Q8_ROWS_MAX = 32;
inline bool q8_rows_applies(long M, bool copies) { return M <= 4 || (copies && M <= Q8_ROWS_MAX); }

}  // namespace tfla
