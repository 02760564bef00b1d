// Which kernel takes a matrix product of the residual block: rules on its sizes alone, by time models of the kernels and measured limits.
// Plain C++ without device code, so that a host program can ask them too.
#pragma once

namespace tfla {

// ---- tiles ------------------------------------------------------------------------------------
struct GemmPlan { int bm, bn, split; double us; };      // us: time by the model

// How a product is cut: the tile and the number of parts with the shortest time by a model of the kernels, measured on products
// of 40 to 8192 rows and columns (forward, both backward layouts; of 160 random ones 2 % above the best of all choices on average,
// 23 % at most).  In us, with w
// workgroups in all, n = ceil(w / 256) of them per CU one after another or side by side, and t steps each:
//   bf16   256 x 256   8 + n (t (1.0 + 0.45 min(1, w / 256)) + 4)        (the power that all CUs draw lowers the clock)
//          256 x 128   7 + n (t (0.63 + 0.31 min(1, w / 256)) + 2)
//          128 x 128   5 + t (0.42 + 0.15 w / 256) up to 256 workgroups, 6 + 0.49 t n + 1.5 max(0, n - 2) above
//          64 x 64     4.8 + 0.177 t n + 0.9 max(0, n - 2)               (pairs: 64 x 128, 0.34 t n)
//   fp32   128 x 128   7 + max(2.3, 2.1 n) t     (steps of 32)
//          64 x 64     5.5 + max(0.68, 0.57 n) t (pairs: 64 x 128, twice that)
//          32 x 32     4.8 + max(0.4, 0.34 n) t  (steps of 64; pairs: 32 x 64, 1.9 times that)
//   joining the parts  4.2 + (bytes written and read again) / 7 MB per us
inline GemmPlan gemm_plan(long M, int N, int K, int segs, int batch, int pair, int dtype) {
    struct Tile { int bm, bn; };
    static constexpr Tile bf16_tiles[] = {{256, 256}, {256, 128}, {128, 128}, {64, 64}}, f32_tiles[] = {{128, 128}, {64, 64}, {32, 32}};
    const bool b16 = dtype == 1;
    const Tile* tiles = b16 ? bf16_tiles : f32_tiles;
    const int kinds = b16 ? 4 : 3;
    GemmPlan best{};
    for (int i = 0; i < kinds; ++i) {
        int bm = tiles[i].bm, bn = tiles[i].bn;
        if (pair && bm <= 64 && bn == bm) bn = 2 * bm;
        const int bno = pair ? bn / 2 : bn;
        const int step = !b16 && bm > 32 ? 32 : 64, all = (K + step - 1) / step * segs;
        const double cells = (double)((M + bm - 1) / bm) * ((N + bno - 1) / bno) * batch;
        for (int split = 1; split <= 32 && (split == 1 || (all >= 4 * split && cells * split <= 1024)); split += split < 4 ? 1 : split / 2) {
            const double w = cells * split, t = (all + split - 1) / split, part = w < 256 ? w / 256 : 1, n = (double)(long)((w + 255) / 256);
            const double more = n > 2 ? n - 2 : 0;
            double us;
            if (!b16) us = bm == 128 ? 7 + (n < 2 ? 2.3 : 2.1 * n) * t : (bm == 64 ? 5.5 + (n < 2 ? 0.68 : 0.57 * n) * t * (pair ? 2 : 1) : 4.8 + (n < 2 ? 0.4 : 0.34 * n) * t * (pair ? 1.9 : 1));
            else if (bn == 256) us = 8 + n * (t * (1.0 + 0.45 * part) + 4);
            else if (bm == 256) us = 7 + n * (t * (0.63 + 0.31 * part) + 2);
            else if (bm == 128) us = n < 2 ? 5 + t * (0.42 + 0.15 * part) : 6 + 0.49 * t * n + 1.5 * more;
            else us = 4.8 + (pair ? 0.34 : 0.177) * t * n + 0.9 * more;
            if (split > 1) us += 4.2 + 8.0 * split * (pair ? 2 : batch) * (double)M * N / 7e6;
            if (best.bm == 0 || us < best.us) best = {bm, bn, split, us};
        }
    }
    return best;
}
// workgroups of a product in one launch
inline long gemm_workgroups(const GemmPlan& p, long M, int N, int batch, int pair) {
    const int bno = pair ? p.bn / 2 : p.bn;
    return ((M + p.bm - 1) / p.bm) * ((N + bno - 1) / bno) * p.split * batch;
}
// Whether some CU gets a second workgroup.  Up to one per CU, tiles of 128 and 64 rows have kernels with more wavefronts and more steps
// under way; the kernels of 256 rows are launched once per CU and take tile after tile.
inline bool gemm_many(long workgroups) { return workgroups > 256; }

// ---- both products of a small backward pass in one launch ------------------------------------------
// dx = dz W and dw = dz^T x in one launch, where gemm_both_applies: both whole, in the same small tiles.  In tiles of 64 x 64 that
// is `items` workgroups with the longest contraction of `longest` steps and `sum` steps in all.
// Tiles of 64 x 128 bring three quarters of the operands' bytes into LDS, which is what bounds these launches, but have half the
// workgroups: taken where the longest of them is at most half of an even share of the steps (2952 x 896 x 3088 65.9 us against
// 82.9, 944 x 1624 x 1360 25.2 against 30.3; with a longest of a whole share 512 x 1024 x 1365, a pair, 26.3 against 22.3).
struct BothSteps {
    long items, longest, sum;
    bool wide() const { return items > 512 && 2 * longest * 256 <= sum; }
};
inline BothSteps both_steps(long M, int K, int N, int pair) {
    auto up = [](long v) { return (v + 63) / 64; };
    const long segs = pair ? 2 : 1, nx = up(M) * up(K), nw = up(N) * up(K) * segs, tx = up(N) * segs, tw = up(M);
    return {nx + nw, tx > tw ? tx : tw, nx * tx + nw * tw};
}
// What a launch costs beside its work (3.4 us of the host's time, 2 of the GPU's) is saved once, and the items of one product fill
// what the other leaves of the CUs' time.  Only of products whose contraction is not divided.  fp32: where both take the same
// small tile.  bf16: by an estimate of the launch of both, fitted as that of single products, against the sum of theirs and 6 us
// (both, one after the other: 1888 x 776 x 2640 39.3, 51.3 us; 368 x 1248 x 2232 20.9, 26.0; 1024 x 4096 x 4096 some 130, 87).
inline bool gemm_both_applies(const GemmPlan& x, const GemmPlan& w, long M, int K, int N, int pair, int dtype) {
    if (x.split != 1 || w.split != 1) return false;
    if (dtype != 1) return x.bm == w.bm && x.bm <= 64;
    const BothSteps b = both_steps(M, K, N, pair);
    const double share = b.sum / 256.0, chain = (b.items > 256 ? 0.4 : 0.2) * b.longest;
    const double us = b.wide() ? 9 + 0.225 * share : 7.5 + (0.29 * share > chain ? 0.29 * share : chain);
    return us <= x.us + w.us + 6;
}

// ---- few rows -----------------------------------------------------------------------------------
constexpr int GEMM_ROWS_MAX = 32;
// Slices where blocks of 16 rows leave CUs without work: fewer than 256, or a last round that is not full (one token through
// 4096 x 4096, 256 blocks: 8.3 us whole, 9.0 in four slices; 684 blocks of a pair: 41.5 and 37.5).
inline int rows_slices(long M, int N) {
    const int n = (N + 15) / 16, rounds = (n + 255) / 256;
    const bool uneven = n < 256 || (rounds < 8 && 256 * rounds * 10 > 11 * n);
    return !uneven || M > 8 ? 1 : (M <= 4 ? 4 : 2);
}
// A lane's registers per piece of 64 contraction steps (in units of those for one bf16 row block), and the pieces that wavefronts have in
// flight.
constexpr int rows_registers(int element_bytes, int row_blocks, bool pair) { return element_bytes / 2 * (row_blocks * (pair ? 2 : 1) < 4 ? 1 : 2); }
constexpr int rows_pieces(int registers, int waves) { return waves > 8 ? 4 / registers : (registers == 4 ? 2 : 4); }
// Wavefronts: as many as leave each of them four pieces, up to eight; sixteen for few blocks with more to read.  Workgroups: one per block of
// 16 / slices rows of weights, or, where a wavefront's share of x fits its registers (hold), as many as the chip runs at a time.
struct RowsPlan { int row_blocks, slices, waves, blocks, grid; bool hold; };
inline RowsPlan rows_plan(long M, int N, int K, bool pair, int element_bytes) {
    RowsPlan p{};
    p.slices = rows_slices(M, N);
    p.row_blocks = M <= 16 ? 1 : 2;
    p.blocks = (N + 16 / p.slices - 1) / (16 / p.slices);
    const int pieces = ((K + 63) / 64 + p.slices - 1) / p.slices;
    p.waves = pieces <= 16 ? 4 : (p.blocks >= 128 || pieces <= 32 ? 8 : 16);
    const int most = 256 * (p.waves <= 4 ? 4 : 2);
    p.hold = p.waves <= 8 && pieces <= p.waves * rows_pieces(rows_registers(element_bytes, p.row_blocks, pair), p.waves) && p.blocks > most;
    p.grid = p.hold ? most : p.blocks;
    return p;
}
// Whether this kernel takes a product or the tiles of gemm_plan do.  Every block of rows reads all of x again, which tiles of 64
// do a quarter as often; tiles need some us more until all CUs have work, and weights that they cannot read in place are
// copied first.  By estimates of both: here rounds of blocks at 27 GB/s per CU (fewer blocks than CUs: 35; fp32 some 10 % less),
// there the plan's time, or the weights at the rate of a copy where that is longer.  Measured, here and there:
// 4096 x 4096, 16 rows 11.8 and 12.2, 32 rows 15.8 and 12.9; pair of 10944 x 4096, 4 rows 38.1 and 39.1, 8 rows 44.9 and 39.5, 32
// rows 62.9 and 40.6; pair of 2752 x 1024, 32 rows 7.5 and 9.3.
inline bool gemm_rows_applies(long M, int N, int K, int pair, int dtype, bool copies) {
    if (M <= 4 || M > GEMM_ROWS_MAX) return M <= 4;
    if (copies) return true;
    const double row = (double)K * (dtype == 1 ? 2 : 4);
    const int rows = 16 / rows_slices(M, N), n = (N + rows - 1) / rows;
    const double rate = (dtype == 1 ? 27e3 : 24e3) * (n < 256 ? 1.3 : 1.0);
    const double here = 1.8 + (n + 255) / 256 * (rows * (pair ? 2 : 1) + M) * row / rate;
    const double there = gemm_plan(M, N, K, 1, 1, pair, dtype).us, read = 5 + (pair ? 2 : 1) * row * N / 5.2e6;
    return here <= (there > read ? there : read);
}

}  // namespace tfla
