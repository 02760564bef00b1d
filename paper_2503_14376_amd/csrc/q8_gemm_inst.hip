// Compiled once per TFLA_Q8 (0: linear, 1: plain results, 2: parts, 3: parts of a pair, 4: a pair's gate): the product kernels in 8 bits
// with that epilogue and their launcher.
#ifndef TFLA_Q8
#error "compile with -DTFLA_Q8=<0..4>"
#endif
#include "q8_wide.h"

namespace tfla {

template <int V> hipError_t launch_q8_gemm_as(const Q8GemmArgs& a, const GemmPlan& p, hipStream_t s);
template <> hipError_t launch_q8_gemm_as<TFLA_Q8>(const Q8GemmArgs& a, const GemmPlan& p, hipStream_t s) {
    constexpr bool PAIR = TFLA_Q8 >= 3;
    constexpr int EPI = TFLA_Q8 == 0 ? EPI_LINEAR : (TFLA_Q8 == 1 ? EPI_STORE : (TFLA_Q8 == 4 ? EPI_GATED : EPI_PART));
    const int bno = PAIR ? p.bn / 2 : p.bn;
    const int tms = (a.g.M + p.bm - 1) / p.bm, tns = (a.g.N + bno - 1) / bno;
    const unsigned n = (unsigned)gemm_workgroups(p, a.g.M, a.g.N, a.g.batch, PAIR);
    // (one workgroup of the wide kernels fits a CU; the 256 of them take the tiles in turn)
    const unsigned wide = n < 256 ? n : 256;
#if TFLA_Q8 == 4
    hipLaunchKernelGGL((gemm_q8_wide_kernel<256, PAIR, EPI>), dim3(wide), dim3(256), 0, s, a, tms, tns);
#else
    const bool many = gemm_many(n);
    if (p.bn == 256) hipLaunchKernelGGL((gemm_q8_wide_kernel<256, PAIR, EPI>), dim3(wide), dim3(256), 0, s, a, tms, tns);
    else if (p.bm == 256) hipLaunchKernelGGL((gemm_q8_wide_kernel<128, PAIR, EPI>), dim3(wide), dim3(256), 0, s, a, tms, tns);
    else if (p.bm == 128) {
        if (many) hipLaunchKernelGGL((gemm_q8_kernel<128, 128, 2, 2, 2, 1, PAIR, EPI>), dim3(n), dim3(256), 0, s, a, tms, tns);
        else hipLaunchKernelGGL((gemm_q8_kernel<128, 128, 4, 2, 4, 1, PAIR, EPI>), dim3(n), dim3(512), 0, s, a, tms, tns);
    } else if constexpr (PAIR) {
        if (many) hipLaunchKernelGGL((gemm_q8_kernel<64, 128, 2, 2, 3, 1, true, EPI>), dim3(n), dim3(256), 0, s, a, tms, tns);
        else hipLaunchKernelGGL((gemm_q8_kernel<64, 128, 2, 2, 3, 2, true, EPI>), dim3(n), dim3(512), 0, s, a, tms, tns);
    } else {
        if (many) hipLaunchKernelGGL((gemm_q8_kernel<64, 64, 2, 2, 3, 1, false, EPI>), dim3(n), dim3(256), 0, s, a, tms, tns);
        else hipLaunchKernelGGL((gemm_q8_kernel<64, 64, 2, 2, 4, 2, false, EPI>), dim3(n), dim3(512), 0, s, a, tms, tns);
    }
#endif
    return hipGetLastError();
}

}  // namespace tfla
