// Products of few rows with a whole matrix of weights (tokens being generated): out(m, n) = sum_k x(m, k) w(n, k), m < 32.
// What bounds them is one read of the weights, so nothing but the loads matters: every wavefront reads 16 rows of w
// straight into the operand registers of v_mfma_f32_16x16x32_bf16 (fp32: 16x16x4), 128 bytes of each row at a time, all of
// its share requested before the first product; the rows of x are the other operand, out of the caches.  The wavefronts of
// a workgroup divide the contraction and meet in LDS.  Rows may start at any address.
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
template <typename DT, int MB, bool PAIR, int EPI, int NW, int U>
__global__ void __launch_bounds__(NW * 64) gemm_rows_kernel(GemmArgs a) {
    constexpr int P = PAIR ? 2 : 1, LD = 20;
    __shared__ __align__(16) float red[NW][P][MB * 16][LD];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4, n0 = blockIdx.x * 16;
    // rows behind the last one read it again: their results are not stored
    const long wrow = (long)min(n0 + r, a.N - 1) * a.ldb + g * 16;
    long xrow[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) xrow[i] = (long)min(i * 16 + r, a.M - 1) * a.lda + g * 16;
    f32x4 acc[P][MB];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < MB; ++i) acc[p][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int full = a.K >> 6, pieces = (a.K + 63) >> 6;
    for (int c0 = wave; c0 < pieces; c0 += NW * U) {
        Vec8<DT> w[U][P][2], x[U][MB][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * NW, k = c * 64;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (c < full) {
#pragma unroll
                    for (int p = 0; p < P; ++p) w[u][p][h].load(a.B[p], wrow + k + h * 8);
#pragma unroll
                    for (int i = 0; i < MB; ++i) x[u][i][h].load(a.A[0], xrow[i] + k + h * 8);
                } else if (c < pieces) {
                    const int left = a.K - k - g * 16 - h * 8;
#pragma unroll
                    for (int p = 0; p < P; ++p) w[u][p][h] = load8<DT>(a.B[p], wrow + k + h * 8, left);
#pragma unroll
                    for (int i = 0; i < MB; ++i) x[u][i][h] = load8<DT>(a.A[0], xrow[i] + k + h * 8, left);
                } else {
#pragma unroll
                    for (int p = 0; p < P; ++p) w[u][p][h].zero();
#pragma unroll
                    for (int i = 0; i < MB; ++i) x[u][i][h].zero();
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int i = 0; i < MB; ++i) acc[p][i] = mma16<DT>(w[u][p][h], x[u][i][h], acc[p][i]);
    }
    // lane (r, g) holds row r of x, columns 4 g ... 4 g + 3
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < MB; ++i) *reinterpret_cast<f32x4*>(&red[wave][p][i * 16 + r][4 * g]) = acc[p][i];
    __syncthreads();
    for (int i = threadIdx.x; i < P * MB * 256; i += NW * 64) {
        const int n = i & 15, m = (i >> 4) % (MB * 16), p = i / (MB * 256);
        float s = red[0][p][m][n];
#pragma unroll
        for (int q = 1; q < NW; ++q) s += red[q][p][m][n];
        red[0][p][m][n] = s;
    }
    __syncthreads();
    const int m = threadIdx.x >> 1, c = (threadIdx.x & 1) * 8;
    if (m < MB * 16) {
        float v[8], u[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { v[e] = red[0][0][m][c + e]; u[e] = PAIR ? red[0][P - 1][m][c + e] : 0.0f; }
        epilogue8<DT, EPI>(a, 0, m, n0 + c, v, u);
    }
}

template <typename DT, int MB, bool PAIR, int EPI> void go(const GemmArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((gemm_rows_kernel<DT, MB, PAIR, EPI, 8, 4>), dim3((a.N + 15) / 16), dim3(512), 0, s, a);
}
template <typename DT> void by_rows(const GemmArgs& a, hipStream_t s) {
    if (a.M <= 16) {
        if (a.pair) go<DT, 1, true, EPI_GATED>(a, s);
        else go<DT, 1, false, EPI_LINEAR>(a, s);
    } else {
        if (a.pair) go<DT, 2, true, EPI_GATED>(a, s);
        else go<DT, 2, false, EPI_LINEAR>(a, s);
    }
}

}  // namespace

hipError_t launch_gemm_rows(const GemmArgs& a, hipStream_t s) {
    if (a.dtype == 1) by_rows<bf16_t>(a, s);
    else by_rows<float>(a, s);
    return hipGetLastError();
}

}  // namespace tfla
