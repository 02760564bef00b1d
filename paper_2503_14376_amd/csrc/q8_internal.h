// Host-side declarations of the residual block in 8 bits: argument blocks and launchers shared by q8_api.hip and the kernels'
// units.  Nothing here is exported.
#pragma once
#include "block_internal.h"
#include "q8_plan.h"

namespace tfla {

// ---- quantisation ------------------------------------------------------------------------------
// Where the codes and scales of a matrix (and of its transpose) go; each pair of pointers may be NULL.
struct Q8Out {
    uint8_t* q; uint8_t* s;            // (M, ldq) codes, (blocks of columns, lds) scales
    uint8_t* qt; uint8_t* st;          // (columns, ldt) codes of the transpose, (blocks of rows, ldst) scales
    // codes of a row (of the transpose) that are stored: the matrix's columns (rows), or more, whose codes are zero
    long ldq, lds, ldt, ldst; int wq, wt;
};
enum { Q8_VALUES = 0, Q8_ACT = 1, Q8_PAIR = 2 };
// One pass over (M, N) values in tiles of 128 x 128: the values themselves (x), dz = x act'(z), or the pair's da = x u act'(z) and
// du = x act(z).  rows = 1: groups of 128 columns of a row, and of 128 rows of a column for the transpose; 128: the tile is the
// group of both.  part: (blocks of rows, 1 or 2, ldp) column sums of the values before rounding, or NULL; with one
// block of rows the sums go to db[0], db[1] instead (each may be NULL).
struct Q8TileArgs {
    const void* x; const void* z; const void* u;
    Q8Out out[2];
    float* part; float* db[2];
    long M; int N; long ldp; int act, dtype, mode, rows;
};
struct Q8RepackArgs;
// b: plain values in the same launch, none where b.M is 0; rp: copies in the same launch
hipError_t launch_q8_tiles(const Q8TileArgs& a, const Q8TileArgs& b, const Q8RepackArgs& rp, hipStream_t s);

// y = norm(x + residual), its codes and scales; sum, y, rstd, mean may be NULL
struct Q8NormArgs : RowNormArgs {
    const void* residual; void* sum; uint8_t* q; uint8_t* s;
};
hipError_t launch_rownorm_q8(const Q8NormArgs& a, hipStream_t s);

// Rows of `cols` bytes at any address -> rows of ldd (a multiple of 16) bytes, zeros behind the columns; up to three matrices.
struct Q8RepackArgs {
    const uint8_t* src[3]; uint8_t* dst[3]; long rows[3];
    int count, cols; long ldd;
    void add(const uint8_t* s, uint8_t* d, long r) { src[count] = s; dst[count] = d; rows[count++] = r; }
};
hipError_t launch_q8_repack(const Q8RepackArgs& a, hipStream_t s);

// ---- products ----------------------------------------------------------------------------------
// out = A B^T of two matrices of codes whose contraction index is the contiguous one.  g: as a product in bf16 whose elements are pairs of
// codes (K, lda, ldb in pairs; pitches multiples of 16 bytes, codes behind the contraction's end zero up to the next
// multiple of 16); k: contraction length in codes.  Scale of row r and block kb of 128: s[kb * ld + (r >> shift)].
struct Q8GemmArgs {
    GemmArgs g;
    const uint8_t* sa[2]; const uint8_t* sb[2];
    long lsa, lsb; int shb;            // (rows of A have a scale each)
    int k;
    Q8Out h; void* hc;                 // EPI_GATED: codes and scales of h; hc: h in bf16 or NULL
};
// (a pair: EPI_GATED where q8_gate_inside, otherwise EPI_PART, which leaves the parts to launch_q8_gated_join)
hipError_t launch_q8_gemm(const Q8GemmArgs& a, const GemmPlan& p, int epi, hipStream_t s);
// column sums of (rows, planes, n) partial sums, in the order of the rows; either result may be NULL
struct Q8Sums { const float* part; int rows, planes, n; float* out[2]; };
struct Q8Both { unsigned first, both; int tms[2], tns[2]; };
// both products of a small backward pass (whole ones, where q8_both_applies) and the sums (planes 0: none) in one launch
hipError_t launch_q8_both(const Q8GemmArgs& x, const Q8GemmArgs& w, const Q8Sums& sums, hipStream_t s);
hipError_t launch_q8_rows(const Q8GemmArgs& a, hipStream_t s);
// h = act(a) u of a pair whose products lie in g.part (split parts of two planes), its codes and scales; stores a, u, h where wanted
hipError_t launch_q8_gated_join(const Q8GemmArgs& a, hipStream_t s);

}  // namespace tfla
