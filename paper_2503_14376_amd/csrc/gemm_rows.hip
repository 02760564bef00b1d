// Products of few rows with a whole matrix of weights (tokens being generated): out(m, n) = sum_k x(m, k) w(n, k), m < 32.
// What bounds them is one read of the weights, so nothing but the loads matters: every wavefront reads 16 rows of w
// straight into the operand registers of v_mfma_f32_16x16x32_bf16 (fp32: 16x16x4), 64 consecutive bytes of each row per access, all of
// its share requested before the first product; the rows of x are the other operand, out of the caches.  The wavefronts of
// a workgroup divide the contraction and meet in LDS.  Rows may start at any address.  One token through 4096 x 4096 in bf16: 8.3 us
// (4.0 TB/s, some 2 us of them before the first load arrives); four through a pair of 10944 x 4096: 38 us (4.7 TB/s).
#include "gemm_epilogue.h"

namespace tfla {

namespace {

template <typename DT> __device__ __forceinline__ f32x4 mma16(const Vec8<DT>& w, const Vec8<DT>& x, f32x4 c);
template <> __device__ __forceinline__ f32x4 mma16<bf16_t>(const Vec8<bf16_t>& w, const Vec8<bf16_t>& x, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w.w), __builtin_bit_cast(bf16x8, x.w), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x4 mma16<float>(const Vec8<float>& w, const Vec8<float>& x, f32x4 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w.v[e], x.v[e], c, 0, 0, 0);
    return c;
}

// MB blocks of 16 rows of x, NW wavefronts, U pieces of 64 contraction steps in flight per wavefront.
// SL slices: with no more than 16 / SL rows of x (MB = 1) the matrix unit's 16 rows and columns are 16 / SL rows of w and x in SL
// slices of the contraction each; of its results those of equal slices count.  A block of work is then 16 / SL rows of w, so
// that there are SL times as many: the CUs are loaded evenly, and matrices of few rows reach more of them.  (One token
// through 512 x 8192: 12.2 us without slices, 6.0 with.)
// HOLD: a wavefront's share of x is no more than U pieces: it stays in registers while the workgroup takes block after block,
// the next block's weights requested before the last one's sums are joined.  (What reaches the CUs in all, 6.2 TB/s, bounds
// the kernel: four tokens through 2 x 10944 x 4096 take 43 us where every four rows of w fetch x anew, 33 where x is one row.)
template <typename DT, int MB, int SL, bool PAIR, int EPI, int NW, int U, bool HOLD>
__global__ void __launch_bounds__(NW * 64) gemm_rows_kernel(GemmArgs a, int blocks) {
    constexpr int P = PAIR ? 2 : 1, RB = 16 / SL, LD = RB + 4;
    static_assert(SL == 1 || MB == 1, "slices take one block of rows");
    __shared__ __align__(16) float red[NW * SL][P][MB * RB][LD];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4, slice = r / RB;
    const int full = a.K >> 6, pieces = (a.K + 63) >> 6, ps = (pieces + SL - 1) / SL;      // ps: pieces of a slice
    long xrow[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) xrow[i] = (long)min(i * 16 + r % RB, a.M - 1) * a.lda + g * 8;
    Vec8<DT> w[U][P][2], x[U][MB][2];
    // piece c0 + u NW of this lane's slice
    auto fetch = [&](int c0, int n0, bool with_w, bool with_x) {
        // rows behind the last one read it again: their results are not stored
        const long wrow = (long)min(n0 + r % RB, a.N - 1) * a.ldb + g * 8;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * NW, k = (slice * ps + c) * 64;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if ((SL - 1) * ps + c < full && c < ps) {
#pragma unroll
                    for (int p = 0; p < P; ++p)
                        if (with_w) w[u][p][h].load(a.B[p], wrow + k + h * 32);
#pragma unroll
                    for (int i = 0; i < MB; ++i)
                        if (with_x) x[u][i][h].load(a.A[0], xrow[i] + k + h * 32);
                } else {
                    const int left = c < ps ? a.K - k - g * 8 - h * 32 : 0;
#pragma unroll
                    for (int p = 0; p < P; ++p)
                        if (with_w) w[u][p][h] = load8<DT>(a.B[p], wrow + k + h * 32, left);
#pragma unroll
                    for (int i = 0; i < MB; ++i)
                        if (with_x) x[u][i][h] = load8<DT>(a.A[0], xrow[i] + k + h * 32, left);
                }
            }
        }
    };
    int block = blockIdx.x;
    if (HOLD) {
        fetch(wave, block * RB, true, false);
        fetch(wave, block * RB, false, true);
    }
    for (; block < blocks; block += gridDim.x) {
        const int n0 = block * RB;
        f32x4 acc[P][MB];
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < MB; ++i) acc[p][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int c0 = wave; c0 < ps || HOLD; c0 += NW * U) {
            if (!HOLD) fetch(c0, n0, true, true);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int i = 0; i < MB; ++i) acc[p][i] = mma16<DT>(w[u][p][h], x[u][i][h], acc[p][i]);
            if (HOLD) break;
        }
        if (HOLD && block + (int)gridDim.x < blocks) fetch(wave, n0 + gridDim.x * RB, true, false);
        // lane (r, g) holds column r (a slice and a row of x) of the rows 4 g ... 4 g + 3 (a slice, four rows of w)
        if (4 * g / RB == slice) {
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < MB; ++i) *reinterpret_cast<f32x4*>(&red[wave * SL + slice][p][i * RB + r % RB][4 * g % RB]) = acc[p][i];
        }
        // (barriers without the fence of __syncthreads, which would wait for the next block's weights)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        for (int i = threadIdx.x; i < P * MB * RB * RB; i += NW * 64) {
            const int n = i % RB, m = i / RB % (MB * RB), p = i / (MB * RB * RB);
            float s = red[0][p][m][n];
#pragma unroll
            for (int q = 1; q < NW * SL; ++q) s += red[q][p][m][n];
            red[0][p][m][n] = s;
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        constexpr int W = RB < 8 ? RB : 8, GR = RB / W;
        const int m = threadIdx.x / GR, c = threadIdx.x % GR * W;
        if (m < MB * RB) {
            float v[8], u[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = e < W ? red[0][0][m][c + e] : 0.0f;
                u[e] = PAIR && e < W ? red[0][P - 1][m][c + e] : 0.0f;
            }
            epilogue8<DT, EPI>(a, 0, m, n0 + c, v, u, W);
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
}

// As many pieces in flight as the wavefronts' registers hold (of eight wavefronts U8, of sixteen U16).
template <typename DT, int MB, int SL, bool PAIR, int EPI, int NW, int U> void launch(const GemmArgs& a, const RowsPlan& p, hipStream_t s) {
    if constexpr (NW <= 8) {
        if (p.hold) {
            hipLaunchKernelGGL((gemm_rows_kernel<DT, MB, SL, PAIR, EPI, NW, U, true>), dim3(p.grid), dim3(NW * 64), 0, s, a, p.blocks);
            return;
        }
    }
    hipLaunchKernelGGL((gemm_rows_kernel<DT, MB, SL, PAIR, EPI, NW, U, false>), dim3(p.grid), dim3(NW * 64), 0, s, a, p.blocks);
}
template <typename DT, int MB, int SL, bool PAIR, int EPI> void go(const GemmArgs& a, const RowsPlan& p, hipStream_t s) {
    constexpr int V = rows_registers(sizeof(DT), MB, PAIR), U8 = rows_pieces(V, 8), U16 = rows_pieces(V, 16);
    if (p.waves == 4) launch<DT, MB, SL, PAIR, EPI, 4, U8>(a, p, s);
    else if (p.waves == 8) launch<DT, MB, SL, PAIR, EPI, 8, U8>(a, p, s);
    else launch<DT, MB, SL, PAIR, EPI, 16, U16>(a, p, s);
}
template <typename DT, bool PAIR, int EPI> void by_rows(const GemmArgs& a, hipStream_t s) {
    const RowsPlan p = rows_plan(a.M, a.N, a.K, PAIR, sizeof(DT));
    if (p.slices == 4) go<DT, 1, 4, PAIR, EPI>(a, p, s);
    else if (p.slices == 2) go<DT, 1, 2, PAIR, EPI>(a, p, s);
    else if (p.row_blocks == 1) go<DT, 1, 1, PAIR, EPI>(a, p, s);
    else go<DT, 2, 1, PAIR, EPI>(a, p, s);
}

}  // namespace

hipError_t launch_gemm_rows(const GemmArgs& a, hipStream_t s) {
    if (a.dtype == 1) {
        if (a.pair) by_rows<bf16_t, true, EPI_GATED>(a, s);
        else by_rows<bf16_t, false, EPI_LINEAR>(a, s);
    } else {
        if (a.pair) by_rows<float, true, EPI_GATED>(a, s);
        else by_rows<float, false, EPI_LINEAR>(a, s);
    }
    return hipGetLastError();
}

}  // namespace tfla
