// Compiled once per TFLA_GEMM (0: both operands plain, 1: B transposed, 2: both transposed, 3: one launch for both products of a
// small backward pass; + 4 for fp32): the product kernels of that layout and their launcher.
#ifndef TFLA_GEMM
#error "compile with -DTFLA_GEMM=<0..7>"
#endif
#include "gemm_wide.h"

namespace tfla {

#if (TFLA_GEMM & 3) != 3

namespace {

template <bool PAIR, int EPI> void go(const GemmArgs& a, const GemmPlan& p, hipStream_t s) {
    constexpr int L = TFLA_GEMM & 3;
    constexpr bool ATR = L == 2, BTR = L >= 1;
    const int bno = PAIR ? p.bn / 2 : p.bn;
    const int tms = (a.M + p.bm - 1) / p.bm, tns = (a.N + bno - 1) / bno;
    const unsigned n = (unsigned)gemm_workgroups(p, a.M, a.N, a.batch, PAIR);
    const bool many = gemm_many(n);
#if TFLA_GEMM >= 4
    // (the pair's tiles cover as many columns of each matrix)
    if (p.bm == 128) hipLaunchKernelGGL((gemm_f32_kernel<128, 128, 2, 2, 1, 32, 1, ATR, BTR, PAIR, EPI>), dim3(n), dim3(256), 0, s, a, tms, tns);
    else if (p.bm == 64) hipLaunchKernelGGL((gemm_f32_kernel<64, PAIR ? 128 : 64, 2, 2, 1, 32, 2, ATR, BTR, PAIR, EPI>), dim3(n), dim3(256), 0, s, a, tms, tns);
    else hipLaunchKernelGGL((gemm_f32_kernel<32, PAIR ? 64 : 32, 1, 1, 4, 64, 1, ATR, BTR, PAIR, EPI>), dim3(n), dim3(256), 0, s, a, tms, tns);
#else
    // (one workgroup of the wide kernels fits a CU; the 256 of them take the tiles in turn)
    if (p.bn == 256) hipLaunchKernelGGL((gemm_bf16_wide_kernel<256, ATR, BTR, PAIR, EPI>), dim3(n < 256 ? n : 256), dim3(256), 0, s, a, tms, tns);
    else if (p.bm == 256) hipLaunchKernelGGL((gemm_bf16_wide_kernel<128, ATR, BTR, PAIR, EPI>), dim3(n < 256 ? n : 256), dim3(256), 0, s, a, tms, tns);
    // 128 x 128: two workgroups on a CU, or one with eight wavefronts and three steps under way instead of one (1024 x 4096 x 4096
    // 64 us with four wavefronts and one step, 46 with three, 44.5 with eight as well)
    else if (p.bm == 128) {
        if (many) hipLaunchKernelGGL((gemm_bf16_kernel<128, 128, 2, 2, 2, 1, ATR, BTR, PAIR, EPI>), dim3(n), dim3(256), 0, s, a, tms, tns);
        else hipLaunchKernelGGL((gemm_bf16_kernel<128, 128, 4, 2, 4, 1, ATR, BTR, PAIR, EPI>), dim3(n), dim3(512), 0, s, a, tms, tns);
    }
    // 64 rows: two groups of wavefronts where no CU gets a second workgroup
    else if constexpr (PAIR) {
        if (many) hipLaunchKernelGGL((gemm_bf16_kernel<64, 128, 2, 2, 3, 1, ATR, BTR, true, EPI>), dim3(n), dim3(256), 0, s, a, tms, tns);
        else hipLaunchKernelGGL((gemm_bf16_kernel<64, 128, 2, 2, 3, 2, ATR, BTR, true, EPI>), dim3(n), dim3(512), 0, s, a, tms, tns);
    } else {
        if (many) hipLaunchKernelGGL((gemm_bf16_kernel<64, 64, 2, 2, 3, 1, ATR, BTR, false, EPI>), dim3(n), dim3(256), 0, s, a, tms, tns);
        else hipLaunchKernelGGL((gemm_bf16_kernel<64, 64, 2, 2, 4, 2, ATR, BTR, false, EPI>), dim3(n), dim3(512), 0, s, a, tms, tns);
    }
#endif
}

}  // namespace

template <int L> hipError_t launch_gemm_layout(const GemmArgs& a, const GemmPlan& p, int epi, hipStream_t s);
template <> hipError_t launch_gemm_layout<TFLA_GEMM>(const GemmArgs& a, const GemmPlan& p, int epi, hipStream_t s) {
#if (TFLA_GEMM & 3) == 0
    if (epi == EPI_PART) {
        if (a.pair) go<true, EPI_PART>(a, p, s);
        else go<false, EPI_PART>(a, p, s);
    } else if (a.pair) go<true, EPI_GATED>(a, p, s);
    else go<false, EPI_LINEAR>(a, p, s);
#else
    if (epi == EPI_PART) go<false, EPI_PART>(a, p, s);
    else go<false, EPI_STORE>(a, p, s);
#endif
    return hipGetLastError();
}

#else

template <int DTYPE> hipError_t launch_gemm_both_as(const GemmArgs& x, const GemmArgs& w, int bm, hipStream_t s);
template <> hipError_t launch_gemm_both_as<TFLA_GEMM == 3>(const GemmArgs& x, const GemmArgs& w, int bm, hipStream_t s) {
    auto up = [](int v, int by) { return (v + by - 1) / by; };
    BothGrid g;
    unsigned all;
    auto cut = [&](int bn) {
        g = {up(x.M, bm), up(x.N, bn), up(w.M, bm), up(w.N, bn), 0, 0};
        g.nx = (unsigned)(g.xms * g.xns);
        const unsigned nw = (unsigned)(g.wms * g.wns * w.batch);
        g.x0 = (long)w.K * w.segs > (long)x.K * x.segs ? nw : 0;
        all = g.nx + nw;
    };
    cut(bm);
#if TFLA_GEMM == 3
    // (up to a workgroup per CU two groups of wavefronts share a tile's steps)
    if (both_steps(x.M, x.N, x.K, x.segs == 2).wide()) {
        cut(128);
        hipLaunchKernelGGL((gemm_bf16_both_kernel<64, 128, 2, 2, 3, 1>), dim3(all), dim3(256), 0, s, x, w, g);
    } else if (gemm_many(all)) hipLaunchKernelGGL((gemm_bf16_both_kernel<64, 64, 2, 2, 3, 1>), dim3(all), dim3(256), 0, s, x, w, g);
    else hipLaunchKernelGGL((gemm_bf16_both_kernel<64, 64, 2, 2, 4, 2>), dim3(all), dim3(512), 0, s, x, w, g);
#else
    if (bm == 64) hipLaunchKernelGGL((gemm_f32_both_kernel<64, 64, 2, 2, 1, 32, 2>), dim3(all), dim3(256), 0, s, x, w, g);
    else hipLaunchKernelGGL((gemm_f32_both_kernel<32, 32, 1, 1, 4, 64, 1>), dim3(all), dim3(256), 0, s, x, w, g);
#endif
    return hipGetLastError();
}

#endif

}  // namespace tfla
