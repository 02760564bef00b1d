// The passes around the matrix products of the residual block: copies into aligned rows, the activation's backward with the
// column sums of the bias gradients, and the join of a contraction that was cut into parts.  All memory-bound: eight
// elements per lane and access (activation of a pair of 8192 x 10944 in bf16: 170 us, 5.3 TB/s).
#include "gemm_epilogue.h"

namespace tfla {

// one instantiation of the products' launcher per operand layout and type (gemm_inst.hip)
template <int L> hipError_t launch_gemm_layout(const GemmArgs& a, const GemmPlan& p, int epi, hipStream_t s);
template <int DTYPE> hipError_t launch_gemm_both_as(const GemmArgs& x, const GemmArgs& w, int bm, hipStream_t s);

namespace {

__global__ void __launch_bounds__(256) repack_kernel(RepackArgs a) {
    const int c = (blockIdx.y * 64 + (threadIdx.x & 63)) * 8, q = blockIdx.z;
    if (c >= a.ldd) return;
    const long step = (long)gridDim.x * 4;
#pragma unroll 4
    for (long r = (long)blockIdx.x * 4 + (threadIdx.x >> 6); r < a.rows[q]; r += step)
        load8<bf16_t>(a.src[q], r * a.cols + c, a.cols - c).store(a.dst[q], r * a.ldd + c);
}

// Workgroups of NW wavefronts: 512 columns, the rows of a row block in turn over the wavefronts.
template <typename DT, bool PAIR, int NW> __global__ void __launch_bounds__(NW * 64) act_bwd_kernel(ActBwdArgs a, int rpb) {
    __shared__ float red[NW][PAIR ? 2 : 1][512];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = (blockIdx.y * 64 + lane) * 8, left = a.N - c;
    const long r0 = (long)blockIdx.x * rpb, r1 = min(a.M, r0 + rpb);
    float s0[8], s1[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { s0[e] = 0.0f; s1[e] = 0.0f; }
    if (c < a.ldd) {
#pragma unroll 2
        for (long r = r0 + wave; r < r1; r += NW) {
            float g[8], z[8], u[8];
            load8<DT>(a.dy, r * a.N + c, left).get(g);
            if (a.z) load8<DT>(a.z, r * a.N + c, left).get(z);
            if constexpr (PAIR) load8<DT>(a.u, r * a.N + c, left).get(u);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (PAIR) {
                    float slope;
                    const float value = act_both<DT>(z[e], a.act, slope), da = g[e] * u[e] * slope;
                    u[e] = g[e] * value;
                    g[e] = da;
                    s1[e] += u[e];
                } else if (a.act != ACT_NONE) {
                    float slope;
                    act_both<DT>(z[e], a.act, slope);
                    g[e] *= slope;
                }
                s0[e] += g[e];
            }
            if (a.dz0) {
                store8<DT>(a.dz0, r * a.ldd + c, 8, g);
                if constexpr (PAIR) store8<DT>(a.dz1, r * a.ldd + c, 8, u);
            }
        }
    }
    if (!a.part && !a.db0 && !a.db1) return;
    store8<float>(red[wave][0], lane * 8, 8, s0);
    if constexpr (PAIR) store8<float>(red[wave][1], lane * 8, 8, s1);
    __syncthreads();
    for (int i = threadIdx.x; i < (PAIR ? 1024 : 512); i += NW * 64) {
        const int p = i >> 9, n = blockIdx.y * 512 + (i & 511);
        if (n >= a.N) continue;
        float s = red[0][p][i & 511];
#pragma unroll
        for (int w = 1; w < NW; ++w) s += red[w][p][i & 511];
        if (a.part) a.part[((long)blockIdx.x * (PAIR ? 2 : 1) + p) * a.ldp + n] = s;
        else if (float* db = p ? a.db1 : a.db0) db[n] = s;
    }
}

// adds the parts of a contraction in order and applies the epilogue, eight columns per lane
template <typename DT, int EPI> __global__ void __launch_bounds__(256) gemm_reduce_kernel(GemmArgs a) {
    const int n = (blockIdx.y * 64 + (threadIdx.x & 63)) * 8;
    const long m = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int b = blockIdx.z, planes = a.pair ? 2 : a.batch;
    if (n >= a.N || m >= a.M) return;
    float v[8], w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { v[e] = 0.0f; w[e] = 0.0f; }
#pragma unroll 4
    for (int p = 0; p < a.split; ++p) {
        float t[8];
        load8<float>(a.part, (((long)p * planes + b) * a.M + m) * a.ld_part + n, 8).get(t);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += t[e];
        if constexpr (EPI == EPI_GATED) {
            load8<float>(a.part, (((long)p * planes + 1) * a.M + m) * a.ld_part + n, 8).get(t);
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] += t[e];
        }
    }
    epilogue8<DT, EPI>(a, b, m, n, v, w);
}

// Rows of a block of the activation's backward: the partial sums stay a small part of the traffic, and a launch has enough
// workgroups to stream.  Up to 32 rows are one block of sixteen wavefronts, whose sums need no second launch.
constexpr int ONE_BLOCK = 32;
int rows_per_block(long M, int N, bool sums) {
    if (sums && M <= ONE_BLOCK) return ONE_BLOCK;
    const long cells = M * ((N + 511) / 512);
    return cells >= 64 * 1024 ? 64 : (cells >= 16 * 512 ? 16 : 4);
}
template <typename DT, bool PAIR> void act_bwd(const ActBwdArgs& a, hipStream_t s) {
    const int rpb = rows_per_block(a.M, a.N, a.part || a.db0 || a.db1);
    const dim3 grid((unsigned)((a.M + rpb - 1) / rpb), (unsigned)((a.ldd + 511) / 512));
    if (rpb == ONE_BLOCK) hipLaunchKernelGGL((act_bwd_kernel<DT, PAIR, 16>), grid, dim3(1024), 0, s, a, rpb);
    else hipLaunchKernelGGL((act_bwd_kernel<DT, PAIR, 4>), grid, dim3(256), 0, s, a, rpb);
}

template <typename DT> hipError_t reduce(const GemmArgs& a, int epi, hipStream_t s) {
    const dim3 grid((unsigned)((a.M + 3) / 4), (a.N + 511) / 512, a.batch), block(256);
    if (epi == EPI_GATED) hipLaunchKernelGGL((gemm_reduce_kernel<DT, EPI_GATED>), grid, block, 0, s, a);
    else if (epi == EPI_LINEAR) hipLaunchKernelGGL((gemm_reduce_kernel<DT, EPI_LINEAR>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((gemm_reduce_kernel<DT, EPI_STORE>), grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_repack(const RepackArgs& a, hipStream_t s) {
    if (a.count == 0) return hipSuccess;
    long most = 1;
    for (int q = 0; q < a.count; ++q) most = a.rows[q] > most ? a.rows[q] : most;
    const long n = (most + 3) / 4;
    const dim3 grid((unsigned)(n < 1024 ? n : 1024), (unsigned)((a.ldd + 511) / 512), a.count);
    hipLaunchKernelGGL(repack_kernel, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

int act_bwd_row_blocks(long M, int N) { const int r = rows_per_block(M, N, true); return (int)((M + r - 1) / r); }

hipError_t launch_act_bwd(const ActBwdArgs& a, hipStream_t s) {
    if (a.dtype == 1) {
        if (a.pair) act_bwd<bf16_t, true>(a, s);
        else act_bwd<bf16_t, false>(a, s);
    } else {
        if (a.pair) act_bwd<float, true>(a, s);
        else act_bwd<float, false>(a, s);
    }
    return hipGetLastError();
}

hipError_t launch_gemm(const GemmArgs& a, const GemmPlan& p, bool a_tr, bool b_tr, int epi, hipStream_t s) {
    const int e = a.split > 1 ? EPI_PART : epi;
    hipError_t rc;
    if (a.dtype == 1) rc = !b_tr ? launch_gemm_layout<0>(a, p, e, s) : (!a_tr ? launch_gemm_layout<1>(a, p, e, s) : launch_gemm_layout<2>(a, p, e, s));
    else rc = !b_tr ? launch_gemm_layout<4>(a, p, e, s) : (!a_tr ? launch_gemm_layout<5>(a, p, e, s) : launch_gemm_layout<6>(a, p, e, s));
    if (rc != hipSuccess || e != EPI_PART) return rc;
    return a.dtype == 1 ? reduce<bf16_t>(a, epi, s) : reduce<float>(a, epi, s);
}

hipError_t launch_gemm_both(const GemmArgs& x, const GemmArgs& w, const GemmPlan& p, hipStream_t s) {
    return x.dtype == 1 ? launch_gemm_both_as<1>(x, w, 64, s) : launch_gemm_both_as<0>(x, w, p.bm, s);
}

}  // namespace tfla
