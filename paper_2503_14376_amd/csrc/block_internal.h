// Host-side declarations of the residual block's operators: row norm, linear projection, gated projection pair.  Argument
// blocks and launchers shared by block_api.hip and the kernels' units.  Nothing here is exported.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>

#include "gemm_plan.h"

namespace tfla {

// ---- norm over D columns ---------------------------------------------------------------------
struct RowNormArgs {
    const void* x; const float* gamma; const float* beta;
    void* y; float* rstd; float* mean;         // rstd, mean: (M) or NULL
    long M; int D, kind, dtype; float eps;
};
struct RowNormBwdArgs {
    const void* x; const void* dy; const float* rstd; const float* mean; const float* gamma; const void* d_residual;
    void* dx;
    // (blocks, 2, D) partial sums of dgamma and dbeta, or NULL: the sums of one block are the results (each may be NULL)
    float* part; float* dgamma; float* dbeta;
    long M; int D, kind, dtype, blocks;
};
int rownorm_bwd_blocks(long M, int D);         // workgroups of the backward launch = partial sums per column
hipError_t launch_rownorm_fwd(const RowNormArgs& a, hipStream_t s);
hipError_t launch_rownorm_bwd(const RowNormBwdArgs& a, hipStream_t s);
// out[j] = sum over r of part[r * rstride + j], j < n, in the order of r; up to two outputs (part + ostride each)
hipError_t launch_sum_rows(const float* part, int rows, long rstride, long ostride, int n, float* out0, float* out1, hipStream_t s);

// ---- matrix products -------------------------------------------------------------------------
// out(i, j) = sum over k of A(i, k) B(j, k).  An operand is "plain" when its contraction index is the contiguous one (rows
// i, columns k) and "transposed" when its rows are k.  Pitches are in elements; base addresses and pitches are multiples of
// 16 bytes, and where the contiguous extent is no multiple of 16 bytes the pitch is larger and the columns in between
// belong to the buffer (zeros where the extent is the contraction's).
enum { EPI_STORE = 0, EPI_LINEAR = 1, EPI_GATED = 2, EPI_PART = 3 };
struct GemmArgs {
    const void* A[2]; const void* B[2];
    long lda, ldb;
    int M, N, K;                 // rows and columns of one output, contraction length of one segment
    // segs = 2: a second pair of operands (A[1], B[1]) whose product is added.  batch = 2: a second product A[1] B[0]^T
    // into out[1].  EPI_GATED (and its EPI_PART): B[0] and B[1] with the same A, both results in one workgroup.
    int segs, batch, pair;
    // epilogue
    const float* bias[2]; const void* residual; void* out[2]; void* z[2];
    int act, dtype;
    // split > 1: the contraction is cut into that many parts, each leaving fp32 partial results in part
    // (split, batch or pair, M, ld_part); gemm_reduce adds them in order and applies the epilogue.
    float* part; long ld_part; int split;
};
// Few rows against plain weights at any address and pitch (forward calls of up to GEMM_ROWS_MAX tokens, where gemm_rows_applies)
hipError_t launch_gemm_rows(const GemmArgs& a, hipStream_t s);
hipError_t launch_gemm(const GemmArgs& a, const GemmPlan& p, bool a_tr, bool b_tr, int epi, hipStream_t s);

// dx = dz W and dw = dz^T x in one launch, where gemm_both_applies: both whole, in the same small tiles
hipError_t launch_gemm_both(const GemmArgs& x, const GemmArgs& w, const GemmPlan& p, hipStream_t s);

// ---- elementwise passes around the products ---------------------------------------------------
// Up to three bf16 matrices of (rows, cols) dense at any address -> rows of ldd elements (zeros behind the columns), in one launch.
struct RepackArgs {
    const void* src[3]; void* dst[3]; long rows[3];
    int count, cols; long ldd;
    void add(const void* s, void* d, long r) { src[count] = s; dst[count] = d; rows[count++] = r; }
};
hipError_t launch_repack(const RepackArgs& a, hipStream_t s);
// Backward of the activation: dz = dy act'(z) (act none: dz = dy), or for the pair da = dh u act'(a), du = dh act(a).
// dz is rounded to the tensors' type, as the matrix unit takes it (bf16: half a step, 2^-8, independent from element to element
// of the sums that follow: relative error of dx and dw 0.0023, 0.0017 by the results' own rounding alone; what the rounding leaves as a second
// operand would double the products' work, 2.3 -> 4.6 ms for a pair of 8192 x 4096 x 10944); the column sums take it before that.
// dz0 / dz1 in rows of ldd elements, zeros behind the columns; dz0 == NULL: sums only.  part: (row blocks, 1 or 2, ldp)
// partial column sums in fp32 of the unrounded values, or NULL; with one row block the sums go to db0, db1 (each may be NULL).
struct ActBwdArgs {
    const void* dy; const void* z; const void* u;
    void* dz0; void* dz1; float* part; float* db0; float* db1;
    long M; int N; long ldd, ldp; int act, dtype, pair;
};
int act_bwd_row_blocks(long M, int N);
hipError_t launch_act_bwd(const ActBwdArgs& a, hipStream_t s);

}  // namespace tfla
